"""The example's projections against their matrices, in 64 bits: queries, keys, values and the block's output of several steps, from the layer's inputs
alone.

Bounds (u = 2^-24): a product of n columns is a sum of n exact products in fp32, scaled by groups or not: off by at most (n + 2 groups) u sum |w x| in
whatever order; it is rounded to fp16 once, and the block's output once more when x is added."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from oracle import decode_oracle as orc
from paper_2406_11674_amd import synth
from test_gpu_decode_layer import example

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HIDDEN, Q_HEADS, KV_HEADS, PAGE, SEED = 512, 8, 2, 16, 3
DIM = HIDDEN // Q_HEADS


def sparse(rows, seed):
    return synth.pruned_fp16(rows, HIDDEN, 0.5, seed=seed).view("float16").astype(np.float64)


def four_bit(rows, seed):
    dense = torch.from_numpy(synth.pruned_fp16(rows, HIDDEN, 1.0, seed=seed).view("float16")).cuda()
    return orc.q4_dense(*(t.cpu().numpy() for t in endor.q4_quantize(dense, 128, zeros=True)), HIDDEN, 128)


def close(got, x, w):
    """Whether fp16 `got` is x w^T as far as its steps go."""
    ref, size = x @ w.T, np.abs(x) @ np.abs(w).T
    off = np.abs(got.astype(np.float64).reshape(ref.shape) - ref)
    fp32 = (HIDDEN + 2 * 4) * U * size
    assert np.all(off <= fp32 + (np.abs(ref) + fp32) * 2.0 ** -11 + 2.0 ** -25), off.max()
    assert np.abs(ref).max() > 0.1
    return ref


def test_the_example():
    layer = example().DecodeLayer(3, hidden=HIDDEN, q_heads=Q_HEADS, kv_heads=KV_HEADS, room=64, budget=40, recent=8, page=PAGE, seed=SEED)
    wq, wo, wk, wv = sparse(HIDDEN, SEED), sparse(HIDDEN, SEED + 1), four_bit(KV_HEADS * DIM, SEED + 2), four_bit(KV_HEADS * DIM, SEED + 3)
    g = torch.Generator(device="cuda").manual_seed(6)
    prompt = torch.randn((3, 20, HIDDEN), generator=g, device="cuda").half()
    layer.prompt(prompt)
    torch.cuda.synchronize()
    table = layer.cache.pages.cpu().numpy()

    def held(pool, b, t):
        return pool[table[b, t // PAGE], :, t % PAGE].reshape(-1).cpu().numpy()

    for b in range(3):
        for t in range(20):
            x = prompt[b, t].double().cpu().numpy()
            close(held(layer.cache.k, b, t), x, wk)
            close(held(layer.cache.v, b, t), x, wv)
    attend, caught = endor.attn_decode, {}

    def attn_decode(cache, q, *args, **kw):
        caught["q"] = q.clone()
        return attend(cache, q, *args, **kw)

    for step in range(12):
        x = torch.randn((3, HIDDEN), generator=g, device="cuda").half()
        endor.attn_decode = attn_decode
        try:
            y = layer.step(x)
        finally:
            endor.attn_decode = attend
        torch.cuda.synchronize()
        xs = x.double().cpu().numpy()
        close(caught["q"].cpu().numpy(), xs, wq)
        for b in range(3):
            close(held(layer.cache.k, b, 20 + step), xs[b], wk)
            close(held(layer.cache.v, b, 20 + step), xs[b], wv)
        out = layer.out.double().cpu().numpy().reshape(3, HIDDEN)
        ref, size = out @ wo.T, np.abs(out) @ np.abs(wo).T
        fp32 = HIDDEN * U * size
        once = fp32 + (np.abs(ref) + fp32) * 2.0 ** -11 + 2.0 ** -25
        off = np.abs(y.double().cpu().numpy() - (xs + ref))
        assert np.all(off <= once + (np.abs(xs + ref) + once) * 2.0 ** -11 + 2.0 ** -25), off.max()
