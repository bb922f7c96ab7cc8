"""The decode side as it is used together: the example's attention block step by step against the oracle, its eviction included, and
steps replayed from a HIP graph while lengths grow on the GPU."""
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
        attend, drop = endor.attn_decode, endor.kv_evict

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
        # the projections, from what the cache was given
        dense = layer.wk.m
        new = np.stack([caught["k"].cpu().numpy()[table[b, lengths[b] // 16], :, lengths[b] % 16] for b in range(3)])
        newv = np.stack([caught["v"].cpu().numpy()[table[b, lengths[b] // 16], :, lengths[b] % 16] for b in range(3)])
        assert dense.rows == 128
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
    assert drop is endor.kv_evict


def state(batch, kv, dim, page, pages, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randperm(batch * pages, generator=g, device="cuda").to(torch.int32).view(batch, pages)
    pool = torch.zeros((2, batch * pages, kv, page, dim), dtype=torch.bfloat16, device="cuda")
    cache = endor.KVCache(pool[0], pool[1], table)
    return {"cache": cache, "pool": pool, "lengths": torch.tensor([0, 17, 300][:batch], dtype=torch.int32, device="cuda"),
            "seen": torch.tensor([0, 17, 300][:batch], dtype=torch.int32, device="cuda"),
            "weights": torch.zeros((batch, kv, cache.capacity), device="cuda"),
            "positions": torch.arange(cache.capacity, dtype=torch.int32, device="cuda").expand(batch, kv, cache.capacity).contiguous(),
            "out": torch.zeros((batch, 4 * kv, dim), dtype=torch.bfloat16, device="cuda"), "lse": torch.zeros((batch, 4 * kv), device="cuda"),
            "x": torch.zeros((batch, 6 * kv, dim), dtype=torch.bfloat16, device="cuda"),
            "scratch": cache.attn_scratch(4 * kv, weights=True), "drop": cache.evict_scratch(310)}


def one_step(s, kv, most):
    q, k, v = s["x"][:, :4 * kv], s["x"][:, 4 * kv:5 * kv], s["x"][:, 5 * kv:]
    endor.kv_append(s["cache"], k, v, s["lengths"], s["seen"], weights=s["weights"], positions=s["positions"], new_lengths=s["lengths"], new_seen=s["seen"])
    endor.attn_decode(s["cache"], q, s["lengths"], max_len=most, weights=s["weights"], new_weights=s["weights"], out=s["out"], lse=s["lse"],
                      scratch=s["scratch"])
    endor.kv_evict(s["cache"], s["lengths"], s["seen"], s["weights"], s["positions"], 310, 16, new_lengths=s["lengths"], new_weights=s["weights"],
                   new_positions=s["positions"], scratch=s["drop"])


@pytest.mark.parametrize("most", [400, 2048], ids=["one launch", "parts"])
def test_steps_in_a_hip_graph(most):
    """Replays with the program's own work and synchronizations in between give what eager calls give, bit for bit, while lengths
    grow and one sequence passes its budget."""
    kv, dim = 2, 64
    eager, graphed = (state(3, kv, dim, 16, 128, 9) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    warm = state(3, kv, dim, 16, 128, 10)
    with torch.cuda.stream(side):
        one_step(warm, kv, most)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        one_step(graphed, kv, most)
    g = torch.Generator(device="cuda").manual_seed(11)
    for step in range(25):
        x = torch.randn(eager["x"].shape, generator=g, device="cuda").bfloat16()
        eager["x"].copy_(x)
        graphed["x"].copy_(x)
        if step % 3 == 0:
            torch.cuda.synchronize()
        one_step(eager, kv, most)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("pool", "lengths", "seen", "weights", "positions", "out", "lse"):
            assert torch.equal(eager[name], graphed[name]), (step, name)
    assert eager["lengths"].tolist() == [25, 42, 310] and eager["seen"].tolist() == [25, 42, 325]
