"""A decoder layer's attention block, token by token, on weights and a cache that are both kept small.

The query and output projections are pruned and stay in the bitmap format, the key and value projections are in 4 bits with
group scales; keys and values go into a paged cache, attention reads it and sums up what each token is attended to, and once a
sequence holds more than `budget` tokens every kv head drops the one that matters least.  Synthetic weights (see
paper_2406_11674_amd/synth.py); the sizes default to a Llama2-70B layer's.

    python examples/decode_layer.py [--batch 4] [--prompt 300] [--steps 64] [--budget 320] [--graph]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2406_11674_amd as endor  # noqa: E402
from paper_2406_11674_amd import synth  # noqa: E402


class Sparse:
    """A pruned projection in the bitmap format: y = x W^T."""

    def __init__(self, rows, cols, batch, seed):
        dense = synth.pruned_fp16(rows, cols, 0.5, seed=seed)
        self.m = endor.to_device(endor.compress(dense))
        self.table, _ = endor.build_offsets(self.m)
        self.y = torch.empty((batch, rows), dtype=torch.float32, device="cuda")
        need = endor.gemm_scratch_bytes(rows, cols, batch)
        self.scratch = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None

    def __call__(self, x):
        return endor.gemm_f16(self.m, self.table, x, Y=self.y, scratch=self.scratch).half()


class FourBit:
    """A quantized projection: codes, a scale and a zero point for every row and group of columns."""

    def __init__(self, rows, cols, batch, seed, group=128):
        dense = torch.from_numpy(synth.pruned_fp16(rows, cols, 1.0, seed=seed).view("float16")).cuda()
        self.m = endor.q4_pack(*endor.q4_quantize(dense, group, zeros=True), cols, group)
        self.y = torch.empty((batch, rows), dtype=torch.float32, device="cuda")
        need = endor.q4_scratch_bytes(self.m, batch)
        self.scratch = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None

    def __call__(self, x):
        return endor.q4_gemm(self.m, x, Y=self.y, scratch=self.scratch).half()


class DecodeLayer:
    """The state of `batch` sequences in one layer.  `room`: the most tokens a sequence holds, prompt included."""

    def __init__(self, batch, hidden=8192, q_heads=64, kv_heads=8, room=384, budget=None, recent=32, page=16, seed=1):
        dim = hidden // q_heads
        self.batch, self.q_heads, self.kv_heads, self.dim, self.budget, self.recent = batch, q_heads, kv_heads, dim, budget, recent
        self.wq, self.wo = Sparse(hidden, hidden, batch, seed), Sparse(hidden, hidden, batch, seed + 1)
        self.wk, self.wv = FourBit(kv_heads * dim, hidden, batch, seed + 2), FourBit(kv_heads * dim, hidden, batch, seed + 3)
        pages = -(-room // page)
        # every sequence's pages lie at random places of the pool, as after some hours of serving
        table = torch.randperm(batch * pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(batch, pages).cuda()
        pool = torch.zeros((2, batch * pages, kv_heads, page, dim), dtype=torch.float16, device="cuda")
        self.cache = endor.KVCache(pool[0], pool[1], table)
        per_slot = (batch, kv_heads, self.cache.capacity)
        self.weights = torch.zeros(per_slot, dtype=torch.float32, device="cuda")
        self.positions = torch.zeros(per_slot, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.seen = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.out = torch.empty((batch, q_heads, dim), dtype=torch.float16, device="cuda")
        self.lse = torch.empty((batch, q_heads), dtype=torch.float32, device="cuda")
        # the host's bound on the lengths: the lengths themselves stay on the GPU
        self.most = min(room, self.cache.capacity) if budget is None else min(budget + 1, self.cache.capacity)
        self.scratch = self.cache.attn_scratch(q_heads, self.cache.capacity, weights=True)
        self.evict_scratch = self.cache.evict_scratch(budget, self.cache.capacity) if budget is not None else None

    def prompt(self, x, counts=None):
        """Keys and values of prompts [batch, tokens, hidden]; sequence b brings counts[b] of the tokens.  No token attends to them yet, so their
        weights are all zero: of a prompt longer than the budget the newest tokens stay, and beside them the first."""
        tokens = x.shape[1]
        k, v = (torch.stack([w(x[:, t].contiguous()) for t in range(tokens)], dim=1).view(self.batch, tokens, self.kv_heads, self.dim)
                for w in (self.wk, self.wv))
        endor.kv_append(self.cache, k, v, self.lengths, self.seen, counts=counts, weights=self.weights, positions=self.positions,
                        new_lengths=self.lengths, new_seen=self.seen)
        self.evict(self.cache.capacity)

    def evict(self, most):
        if self.budget is not None:
            endor.kv_evict(self.cache, self.lengths, self.seen, self.weights, self.positions, self.budget, self.recent, max_len=most,
                           new_lengths=self.lengths, new_weights=self.weights, new_positions=self.positions, scratch=self.evict_scratch)

    def step(self, x):
        """One token of every sequence, x [batch, hidden] float16; returns the block's output.  Everything is enqueued, nothing waited for."""
        q = self.wq(x).view(self.batch, self.q_heads, self.dim)
        k, v = (w(x).view(self.batch, self.kv_heads, self.dim) for w in (self.wk, self.wv))
        endor.kv_append(self.cache, k, v, self.lengths, self.seen, weights=self.weights, positions=self.positions, new_lengths=self.lengths,
                        new_seen=self.seen)
        endor.attn_decode(self.cache, q, self.lengths, max_len=self.most, weights=self.weights, new_weights=self.weights, out=self.out,
                          lse=self.lse, scratch=self.scratch)
        self.evict(self.most)
        return x + self.wo(self.out.view(self.batch, -1))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 4), ("prompt", 300), ("steps", 64), ("budget", 320), ("hidden", 8192), ("q-heads", 64), ("kv-heads", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--graph", action="store_true", help="capture a step into a HIP graph and replay it")
    a = ap.parse_args()
    layer = DecodeLayer(a.batch, a.hidden, a.q_heads, a.kv_heads, room=max(a.prompt, a.budget) + 1, budget=a.budget)
    g = torch.Generator(device="cuda").manual_seed(7)
    layer.prompt(torch.randn((a.batch, a.prompt, a.hidden), generator=g, device="cuda").half())
    x = torch.randn((a.batch, a.hidden), generator=g, device="cuda").half()
    run = lambda: x.copy_(torch.nn.functional.layer_norm(layer.step(x).float(), (a.hidden,)).half())  # noqa: E731
    run()
    if a.graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        run = graph.replay
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.steps):
        run()
    torch.cuda.synchronize()
    us = (time.perf_counter() - began) / a.steps * 1e6
    print("%d sequences, %d tokens each held after %d seen: %.1f us a token and layer (attention block)"
          % (a.batch, int(layer.lengths[0]), int(layer.seen[0]), us))


if __name__ == "__main__":
    main()
