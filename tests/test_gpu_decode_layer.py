"""The decode side as it is used together: the example's attention block step by step against the oracle, its eviction included."""
import importlib.util
import os

import numpy as np
import pytest

import paper_2406_11674_amd as endor
from oracle import decode_oracle as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decode_layer", os.path.join(ROOT, "examples", "decode_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_against_the_oracle():
    """Projections against their dense forms, then the cache, the attention and the eviction of every step against the oracle's on the same
    queries, keys and values; the weights that eviction goes by are the GPU's, so it has to agree exactly."""
    layer = example().DecodeLayer(3, hidden=512, q_heads=8, kv_heads=2, room=64, budget=40, recent=8, page=16, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    layer.prompt(torch.randn((3, 50, 512), generator=g, device="cuda").half(), counts=torch.tensor([50, 0, 20], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert layer.lengths.tolist() == [40, 0, 20] and layer.seen.tolist() == [50, 0, 20]
    table = layer.cache.pages.cpu().numpy()
    for step in range(30):
        k, v = layer.cache.k.cpu().numpy().copy(), layer.cache.v.cpu().numpy().copy()
        lengths, seen = layer.lengths.cpu().numpy(), layer.seen.cpu().numpy()
        w, pos = layer.weights.cpu().numpy().copy(), layer.positions.cpu().numpy().copy()
        x = torch.randn((3, 512), generator=g, device="cuda").half()
        caught = {}
        attend = endor.attn_decode

        def attn_decode(cache, q, *args, **kw):
            caught["q"] = q.clone()
            result = attend(cache, q, *args, **kw)
            caught["weights"] = kw["new_weights"].clone()
            caught["k"], caught["v"] = cache.k.clone(), cache.v.clone()
            return result

        endor.attn_decode = attn_decode
        try:
            y = layer.step(x)
        finally:
            endor.attn_decode = attend
        torch.cuda.synchronize()
        q = caught["q"]
        # the key projection, from what the cache was given
        new = np.stack([caught["k"].cpu().numpy()[table[b, lengths[b] // 16], :, lengths[b] % 16] for b in range(3)])
        newv = np.stack([caught["v"].cpu().numpy()[table[b, lengths[b] // 16], :, lengths[b] % 16] for b in range(3)])
        ref_k = endor.q4_gemm(layer.wk.m, x).half().view(3, 2, 64).cpu().numpy()
        assert np.array_equal(new, ref_k)
        lengths, seen = orc.append(k, v, table, lengths, seen, new[:, None], newv[:, None], None, w, pos)
        assert np.array_equal(caught["k"].cpu().numpy(), k) and np.array_equal(caught["v"].cpu().numpy(), v)
        ref, _, probs, _, _ = orc.attention(k, v, table, q.cpu().numpy(), lengths, 41, 64 ** -0.5)
        assert np.abs(layer.out.float().cpu().numpy() - ref).max() < 2e-3
        got = caught["weights"].cpu().numpy()
        for b in range(3):
            slots, p = probs[b]
            for h in range(8):
                w[b, h // 4, slots] += p[h]
            assert np.abs(got[b, :, :lengths[b]] - w[b, :, :lengths[b]]).max() < 1e-4
        w = got.copy()
        after = orc.evict(k, v, table, lengths, seen, w, pos, 40, 8, 41)
        assert np.array_equal(layer.lengths.cpu().numpy(), after) and np.array_equal(layer.seen.cpu().numpy(), seen)
        assert np.array_equal(layer.cache.k.cpu().numpy(), k) and np.array_equal(layer.cache.v.cpu().numpy(), v)
        for b in range(3):
            assert np.array_equal(layer.weights.cpu().numpy()[b, :, :after[b]], w[b, :, :after[b]])
            assert np.array_equal(layer.positions.cpu().numpy()[b, :, :after[b]], pos[b, :, :after[b]])
        assert torch.isfinite(y.float()).all()
