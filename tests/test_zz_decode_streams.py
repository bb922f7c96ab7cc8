"""The decode side on streams of its own and in a HIP graph.  Collected after the pipeline's timing test: how well that one's copies overlap
depends on which streams of torch's pool it gets, and this file takes some."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from test_gpu_attn_decode import make as make_cache
from test_gpu_q4 import make as make_q4

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_attention_same_from_run_to_run_and_on_another_stream():
    lengths = [3000, 17, 900]
    cache, q, k, v, table = make_cache(lengths, (32, 4), 128, 16, torch.bfloat16, seed=14)
    qd, lens = q.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    first = endor.attn_decode(cache, qd, lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    scratch = cache.attn_scratch(32)
    with torch.cuda.stream(side):
        torch.cuda._sleep(1000000)
        late = qd * 1  # made on the side stream after a while
        second = endor.attn_decode(cache, late, lens, scratch=scratch)
    side.synchronize()
    third = endor.attn_decode(cache, qd, lens, stream=side)
    side.synchronize()
    for other in (second, third):
        assert torch.equal(first[0], other[0]) and torch.equal(first[1], other[1])


def test_q4_same_from_run_to_run_and_on_another_stream():
    m, w, g = make_q4(300, 5000, 128, True, seed=6)
    x = torch.from_numpy(g.standard_normal((16, 5000), dtype=np.float32)).half().cuda()
    a = endor.q4_gemm(m, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = endor.q4_gemm(m, x, stream=side)
    side.synchronize()
    assert torch.equal(a, b)


def test_what_a_call_allocates_belongs_to_its_stream():
    """Outputs, scratch and copies that a call makes for itself on a side stream, while the current stream is busy and takes and
    returns memory of the same sizes."""
    lengths = [3000, 17, 900]
    cache, q, k, v, table = make_cache(lengths, (32, 4), 128, 16, torch.bfloat16, seed=14)
    qd, lens = q.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    w = torch.rand((3, 4, cache.capacity), device="cuda")
    pos = torch.arange(cache.capacity, dtype=torch.int32, device="cuda").expand(3, 4, cache.capacity).contiguous()
    want = endor.kv_evict(endor.KVCache(cache.k.clone(), cache.v.clone(), cache.pages), lens, lens, w, pos, 500, 9)
    out = torch.empty_like(qd), torch.empty((3, 32), device="cuda"), torch.empty_like(w)
    endor.attn_decode(cache, qd, lens, weights=w, new_weights=out[2], out=out[0], lse=out[1])
    m, _, g = make_q4(64, 60000, 128, True, seed=8)   # its columns are split
    x = torch.from_numpy(g.standard_normal((4, 60000), dtype=np.float32)).half().cuda()
    y = endor.q4_gemm(m, x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        torch.cuda._sleep(2000000)                     # the current stream is behind the side stream
        junk = [torch.full((n,), float("nan"), device="cuda") for n in (3 * 4 * cache.capacity, 1 << 20, 3 * 32 * 128, 3, 96)]
        del junk
        again = endor.q4_gemm(m, x, stream=side)
        got = torch.zeros_like(out[2])
        side.wait_stream(torch.cuda.current_stream())
        o, lse = endor.attn_decode(cache, qd, lens, weights=w, new_weights=got, stream=side)
        evicted = endor.kv_evict(endor.KVCache(cache.k.clone(), cache.v.clone(), cache.pages), lens, lens, w, pos, 500, 9, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(again, y) and torch.equal(o, out[0]) and torch.equal(lse, out[1])
        for b, n in enumerate(lengths):
            assert torch.equal(got[b, :, :n], out[2][b, :, :n])
        assert torch.equal(evicted[0], want[0])
        for a, z in zip(evicted[1:], want[1:]):
            assert torch.equal(a, z)


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
