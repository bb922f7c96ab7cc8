"""A batch of no sequences is work that is done, at every entry point and for every bound on the lengths."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_2406_11674_amd as endor
from paper_2406_11674_amd import decode

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def sizes():
    c = decode._Cache()
    c.d_k = c.d_v = c.d_pages = 0x10000  # never looked at
    c.page_stride, c.head_stride, c.slot_stride, c.num_pages, c.pages_stride = 4096, 1024, 64, 10, 1 << 12
    c.batch, c.kv_heads, c.head_dim, c.page_size, c.max_pages, c.dtype = 0, 2, 64, 16, 1 << 12, 0
    L, at = decode._lib(), ctypes.addressof(c)
    got = [L.endor_attn_scratch_bytes(at, heads, most, weights) for heads in (2, 4, 64) for most in (0, 1, 1024, 1025, 1 << 16, 1 << 30) for weights in (0, 1)]
    return got + [L.endor_kv_evict_scratch_bytes(at, budget, 1 << 16) for budget in (0, 1, 1000)]


def test_no_scratch():
    """In a process of its own, for a division by the number of sequences ends one."""
    code = "import sys; sys.path[:0] = [%r, %r]; import test_decode_empty_batch as t; assert not any(t.sizes()); print('none')"
    proc = subprocess.run([sys.executable, "-c", code % (ROOT, os.path.join(ROOT, "tests"))], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert proc.returncode == 0 and proc.stdout.strip().endswith("none"), proc.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("pages", [0, 1, 4096])
def test_calls(pages):
    pool = torch.zeros((2, 3, 2, 16, 64), dtype=torch.float16, device="cuda")
    cache = endor.KVCache(pool[0], pool[1], torch.zeros((0, pages), dtype=torch.int32, device="cuda"))
    lengths, new = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros((0, 2, 64), dtype=torch.float16, device="cuda")
    w, pos = torch.zeros((0, 2, cache.capacity), device="cuda"), torch.zeros((0, 2, cache.capacity), dtype=torch.int32, device="cuda")
    n, seen = endor.kv_append(cache, new, new, lengths, weights=w, positions=pos)
    out, lse = endor.attn_decode(cache, torch.zeros((0, 8, 64), dtype=torch.float16, device="cuda"), lengths, weights=w, new_weights=w)
    after, _, _ = endor.kv_evict(cache, lengths, lengths, w, pos, 8, 2)
    assert n.shape == seen.shape == after.shape == (0,) and out.shape == (0, 8, 64) and lse.shape == (0, 8)
    assert torch.all(pool == 0)
