"""The decode side: a paged key-value cache with the attention that reads it, eviction from it, and products with
4-bit weights.  Argument marshalling over include/endor.h, as in `binding`; every step runs inside libendor.so."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

from . import binding
from .binding import _check, _dptr, _i64, _p, _stream_handle, _sz, _torch

__all__ = ["KVCache", "kv_append", "attn_decode", "kv_evict", "Q4Matrix", "q4_pack", "q4_quantize", "q4_scratch_bytes", "q4_gemm"]

_i32 = ctypes.c_int32


class _Cache(ctypes.Structure):
    _fields_ = [("d_k", _p), ("d_v", _p), ("page_stride", _i64), ("head_stride", _i64), ("slot_stride", _i64),
                ("num_pages", _i64), ("d_pages", _p), ("pages_stride", _i64), ("batch", _i32), ("kv_heads", _i32),
                ("head_dim", _i32), ("page_size", _i32), ("max_pages", _i32), ("dtype", _i32)]


_declared = None


def _lib():
    global _declared
    L = binding.lib()
    if _declared is not L:
        L.endor_kv_append.argtypes = [_p, _p, _p, _i64, _i64, _i64, ctypes.c_int, _p, _p, _p, _p, _p, _p, _p, _p]
        L.endor_attn_scratch_bytes.restype = _sz
        L.endor_attn_scratch_bytes.argtypes = [_p, ctypes.c_int, _i32, ctypes.c_int]
        L.endor_attn_decode.argtypes = [_p, ctypes.c_int, _p, _i64, _i64, _p, _i32, _p, _i64, ctypes.c_float, _p, _p, _p, _p, _p, _sz, _p]
        L.endor_kv_evict_scratch_bytes.restype = _sz
        L.endor_kv_evict_scratch_bytes.argtypes = [_p, _i32, _i32]
        L.endor_kv_evict.argtypes = [_p, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _p]
        L.endor_q4_bytes.restype = _sz
        L.endor_q4_bytes.argtypes = [_i64, _i64, ctypes.c_int, ctypes.c_int]
        L.endor_q4_pack.argtypes = [_i64, _i64, ctypes.c_int, _p, _p, _p, _p, _sz, _p]
        L.endor_q4_quantize.argtypes = [_i64, _i64, ctypes.c_int, _p, _p, _p, _p, _p]
        L.endor_q4_scratch_bytes.restype = _sz
        L.endor_q4_scratch_bytes.argtypes = [_i64, _i64, ctypes.c_int, ctypes.c_int]
        L.endor_q4_gemm.argtypes = [_i64, _i64, ctypes.c_int, ctypes.c_int, _p, _sz, ctypes.c_int, _p, _i64, ctypes.c_int, _p, _p, _sz, _p]
        _declared = L
    return L


def _dtype_code(dtype):
    torch = _torch()
    if dtype == torch.float16:
        return 0
    if dtype == torch.bfloat16:
        return 1
    raise ValueError("elements are float16 or bfloat16, got %s" % dtype)


def _on(device, *tensors):
    """All of the tensors that a kernel is to reach lie on that GPU."""
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on the cache's (the weight's) GPU")


def _ints(t, count, name):
    torch = _torch()
    if t.dtype != torch.int32 or t.numel() != count or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of %d elements" % (name, count))
    return t


class KVCache:
    """A paged cache: k and v are pools of pages [pages, kv_heads, page_size, head_dim] (any strides whose last is 1 and
    whose others are multiples of 8 elements; the same for both), `pages` the int32 table [batch, max_pages] of every
    sequence's pages.  The tensors stay the caller's: what they hold may change between calls, the tensors may not."""

    def __init__(self, k, v, pages):
        torch = _torch()
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.device != pages.device:
            raise ValueError("k and v must be alike, [pages, kv_heads, page_size, head_dim], on the table's device")
        if pages.dtype != torch.int32 or pages.dim() != 2 or (pages.shape[1] > 1 and pages.stride(1) != 1):
            raise ValueError("pages must be an int32 tensor [batch, max_pages] with contiguous rows")
        if any(n > 1 and a != b for n, a, b in zip(k.shape, k.stride(), v.stride())) or (k.shape[3] > 1 and k.stride(3) != 1):
            raise ValueError("k and v must have the same strides, the last one 1")
        if not k.is_cuda:
            raise ValueError("the cache lies in GPU memory")
        self.k, self.v, self.pages, self.device_index = k, v, pages, k.get_device()
        self.num_pages, self.kv_heads, self.page_size, self.head_dim = (int(n) for n in k.shape)
        self.batch, self.max_pages = int(pages.shape[0]), int(pages.shape[1])
        self.capacity = self.max_pages * self.page_size
        c = self._c = _Cache()
        c.d_k, c.d_v, c.d_pages = _dptr(k), _dptr(v), _dptr(pages)
        # the stride over a dimension of one element is never used, whatever torch says it is
        c.page_stride, c.head_stride, c.slot_stride = (int(k.stride(i)) if k.shape[i] > 1 else -(-self.head_dim // 8) * 8 for i in range(3))
        c.num_pages, c.pages_stride = self.num_pages, int(pages.stride(0)) if self.batch > 1 else self.max_pages
        c.batch, c.kv_heads, c.head_dim, c.page_size, c.max_pages = self.batch, self.kv_heads, self.head_dim, self.page_size, self.max_pages
        c.dtype = _dtype_code(k.dtype)
        self._at = ctypes.addressof(c)

    def _scratch(self, nbytes):
        return _torch().empty(nbytes, dtype=_torch().uint8, device=self.k.device) if nbytes else None

    def attn_scratch(self, q_heads, max_len=None, weights=False):
        """Scratch of attn_decode for calls with these bounds; None if it takes none.  Calls that overlap in time need distinct ones."""
        return self._scratch(_lib().endor_attn_scratch_bytes(self._at, q_heads, self.capacity if max_len is None else max_len, int(weights)))

    def evict_scratch(self, budget, max_len=None):
        """Scratch of kv_evict, likewise."""
        return self._scratch(_lib().endor_kv_evict_scratch_bytes(self._at, budget, self.capacity if max_len is None else max_len))

    def _per_slot(self, t, name, dtype):
        if t.dtype != dtype or t.shape != (self.batch, self.kv_heads, self.capacity) or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor [batch, kv_heads, capacity]" % (name, dtype))
        return t


def kv_append(cache, k, v, lengths, seen=None, counts=None, weights=None, positions=None, new_lengths=None, new_seen=None, stream=None):
    """endor_kv_append.  k, v: [batch, tokens, kv_heads, head_dim], or without `tokens` for one each.  `seen` defaults to
    `lengths` (nothing was evicted).  Returns (new_lengths, new_seen); pass lengths and seen for them to advance in place."""
    torch = _torch()
    if k.dim() == 3:
        k, v = k.unsqueeze(1), v.unsqueeze(1)
    batch, tokens = cache.batch, int(k.shape[1])
    if tuple(k.shape) != (batch, tokens, cache.kv_heads, cache.head_dim) or k.shape != v.shape or k.dtype != cache.k.dtype or v.dtype != k.dtype:
        raise ValueError("k and v must be [batch, tokens, kv_heads, head_dim] of the cache's type")
    if k.stride() != v.stride():
        v = v.contiguous()
        k = k.contiguous()
    if k.stride(3) != 1 and cache.head_dim > 1:
        raise ValueError("the last stride of k and v must be 1")
    _ints(lengths, batch, "lengths")
    seen = lengths if seen is None else _ints(seen, batch, "seen")
    if counts is not None:
        _ints(counts, batch, "counts")
    if weights is not None:
        cache._per_slot(weights, "weights", torch.float32)
    if positions is not None:
        cache._per_slot(positions, "positions", torch.int32)
    new_lengths = torch.empty_like(lengths) if new_lengths is None else _ints(new_lengths, batch, "new_lengths")
    new_seen = torch.empty_like(seen) if new_seen is None else _ints(new_seen, batch, "new_seen")
    _on(cache.device_index, k, v, lengths, seen, counts, weights, positions, new_lengths, new_seen)
    st = k.stride()
    _check(_lib().endor_kv_append(cache._at, _dptr(k), _dptr(v), st[0], st[1], st[2], tokens, _dptr(counts), _dptr(lengths), _dptr(seen),
                                  _dptr(new_lengths), _dptr(new_seen), _dptr(weights), _dptr(positions), _stream_handle(stream)),
           "endor_kv_append")
    return new_lengths, new_seen


def attn_decode(cache, q, lengths, max_len=None, mask=None, scale=None, weights=None, new_weights=None, out=None, lse=None, scratch=None,
                stream=None):
    """endor_attn_decode.  q: [batch, q_heads, head_dim] of the cache's type; lengths: int32 [batch] on the device; max_len: the host's
    bound on them (default: the capacity); mask: int64 words [batch, >= ceil(max_len / 64)], a 0 bit hides its slot; scale defaults
    to head_dim ** -0.5.  With new_weights the tokens' attention weights are added to `weights` (None: to 0) into it.
    Returns (out, lse)."""
    torch = _torch()
    batch, max_len = cache.batch, cache.capacity if max_len is None else int(max_len)
    if q.dim() != 3 or q.shape[0] != batch or q.shape[2] != cache.head_dim or q.dtype != cache.k.dtype or (cache.head_dim > 1 and q.stride(2) != 1):
        raise ValueError("q must be [batch, q_heads, head_dim] of the cache's type, its last stride 1")
    q_heads = int(q.shape[1])
    _ints(lengths, batch, "lengths")
    mask_stride = 0
    if mask is not None:
        words = (min(max_len, cache.capacity) + 63) // 64
        if mask.dtype != torch.int64 or mask.dim() != 2 or mask.shape[0] != batch or mask.shape[1] < words or (mask.shape[1] > 1 and mask.stride(1) != 1):
            raise ValueError("mask must be an int64 tensor [batch, >= %d] with contiguous rows" % words)
        mask_stride = int(mask.stride(0))
    if weights is not None:
        cache._per_slot(weights, "weights", torch.float32)
        if new_weights is None:
            raise ValueError("weights without new_weights: pass the buffer for the sums, which may be weights itself")
    if new_weights is not None:
        cache._per_slot(new_weights, "new_weights", torch.float32)
    if out is None:
        out = torch.empty((batch, q_heads, cache.head_dim), dtype=q.dtype, device=q.device)
    elif out.dtype != q.dtype or out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor like q")
    if lse is None:
        lse = torch.empty((batch, q_heads), dtype=torch.float32, device=q.device)
    elif lse.dtype != torch.float32 or lse.numel() != batch * q_heads or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor [batch, q_heads]")
    if scratch is None:
        scratch = cache.attn_scratch(q_heads, max_len, new_weights is not None)
    _on(cache.device_index, q, lengths, mask, weights, new_weights, out, lse, scratch)
    _check(_lib().endor_attn_decode(cache._at, q_heads, _dptr(q), q.stride(0), q.stride(1), _dptr(lengths), max_len, _dptr(mask), mask_stride,
                                    cache.head_dim ** -0.5 if scale is None else scale, _dptr(out), _dptr(lse), _dptr(weights),
                                    _dptr(new_weights), _dptr(scratch), 0 if scratch is None else scratch.numel(), _stream_handle(stream)),
           "endor_attn_decode")
    return out, lse


def kv_evict(cache, lengths, seen, weights, positions, budget, recent, max_len=None, new_lengths=None, new_weights=None, new_positions=None,
             scratch=None, stream=None):
    """endor_kv_evict: every kv head of every sequence keeps `budget` tokens, the newest `recent` and those of the largest weight.
    Returns (new_lengths, new_weights, new_positions); pass the inputs for them to change in place."""
    torch = _torch()
    max_len = cache.capacity if max_len is None else int(max_len)
    _ints(lengths, cache.batch, "lengths")
    _ints(seen, cache.batch, "seen")
    cache._per_slot(weights, "weights", torch.float32)
    cache._per_slot(positions, "positions", torch.int32)
    new_lengths = torch.empty_like(lengths) if new_lengths is None else _ints(new_lengths, cache.batch, "new_lengths")
    new_weights = torch.zeros_like(weights) if new_weights is None else cache._per_slot(new_weights, "new_weights", torch.float32)
    new_positions = torch.zeros_like(positions) if new_positions is None else cache._per_slot(new_positions, "new_positions", torch.int32)
    if scratch is None:
        scratch = cache.evict_scratch(budget, max_len)
    _on(cache.device_index, lengths, seen, weights, positions, new_lengths, new_weights, new_positions, scratch)
    _check(_lib().endor_kv_evict(cache._at, budget, recent, max_len, _dptr(lengths), _dptr(seen), _dptr(weights), _dptr(positions),
                                 _dptr(new_lengths), _dptr(new_weights), _dptr(new_positions), _dptr(scratch),
                                 0 if scratch is None else scratch.numel(), _stream_handle(stream)), "endor_kv_evict")
    return new_lengths, new_weights, new_positions


# ------------------------------------------------------------------ 4-bit weights

@dataclass
class Q4Matrix:
    """A 4-bit weight in the form the products read (device memory)."""
    rows: int
    cols: int
    group: int
    zeros: bool     # whether it has zero points of its own
    packed: object  # torch.uint8


def _q4_groups(cols, group):
    return -(-cols // group)


def q4_pack(codes, scales, zeros, cols, group, stream=None):
    """endor_q4_pack.  codes: uint8 [rows, (cols + 1) // 2], the even column in the low half; scales: float16 [rows, ceil(cols / group)];
    zeros: uint8 of that shape, or None for 8 everywhere.  Returns a Q4Matrix."""
    torch = _torch()
    if group < 1:
        raise ValueError("group must be a power of two from 32 on")
    rows = int(codes.shape[0])
    if codes.dtype != torch.uint8 or tuple(codes.shape) != (rows, (cols + 1) // 2) or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous uint8 tensor [rows, (cols + 1) // 2]")
    shape = (rows, _q4_groups(cols, group))
    if scales.dtype != torch.float16 or tuple(scales.shape) != shape or not scales.is_contiguous():
        raise ValueError("scales must be a contiguous float16 tensor [rows, ceil(cols / group)]")
    if zeros is not None and (zeros.dtype != torch.uint8 or tuple(zeros.shape) != shape or not zeros.is_contiguous()):
        raise ValueError("zeros must be a contiguous uint8 tensor [rows, ceil(cols / group)]")
    if not codes.is_cuda:
        raise ValueError("codes must lie in GPU memory")
    _on(codes.get_device(), scales, zeros)
    L = _lib()
    packed = torch.empty(L.endor_q4_bytes(rows, cols, group, int(zeros is not None)), dtype=torch.uint8, device=codes.device)
    _check(L.endor_q4_pack(rows, cols, group, _dptr(codes), _dptr(scales), _dptr(zeros), _dptr(packed), packed.numel(), _stream_handle(stream)),
           "endor_q4_pack")
    return Q4Matrix(rows, cols, group, zeros is not None, packed)


def q4_quantize(dense, group=128, zeros=False, stream=None):
    """endor_q4_quantize on a contiguous 2-d float16 tensor.  Returns (codes, scales, zeros or None), as q4_pack takes them."""
    torch = _torch()
    if dense.dtype != torch.float16 or dense.dim() != 2 or not dense.is_contiguous():
        raise ValueError("dense must be a contiguous 2-d float16 tensor")
    rows, cols = (int(n) for n in dense.shape)
    if not dense.is_cuda:
        raise ValueError("dense must lie in GPU memory")
    if group < 1:
        raise ValueError("group must be a power of two from 32 on")
    codes = torch.empty((rows, (cols + 1) // 2), dtype=torch.uint8, device=dense.device)
    scales = torch.empty((rows, _q4_groups(cols, group)), dtype=torch.float16, device=dense.device)
    points = torch.empty(scales.shape, dtype=torch.uint8, device=dense.device) if zeros else None
    _check(_lib().endor_q4_quantize(rows, cols, group, _dptr(dense), _dptr(codes), _dptr(scales), _dptr(points), _stream_handle(stream)),
           "endor_q4_quantize")
    return codes, scales, points


def q4_scratch_bytes(m, nb):
    """endor_q4_scratch_bytes: scratch of q4_gemm with that many right-hand sides; mostly none."""
    return int(_lib().endor_q4_scratch_bytes(m.rows, m.cols, m.group, nb))


def q4_gemm(m, X, Y=None, scratch=None, stream=None):
    """endor_q4_gemm: Y (fp32, nb x rows) = X W^T; X: (nb, cols) float16 or bfloat16 (row stride = ldx), nb <= 16."""
    torch = _torch()
    if X.dim() != 2 or X.shape[1] != m.cols or (m.cols > 1 and X.stride(1) != 1):
        raise ValueError("X must be (nb, cols) with contiguous rows")
    nb = int(X.shape[0])
    if Y is None:
        Y = torch.empty((nb, m.rows), dtype=torch.float32, device=X.device)
    elif Y.dtype != torch.float32 or Y.numel() != nb * m.rows or not Y.is_contiguous():
        raise ValueError("Y must be a contiguous fp32 tensor of nb*rows elements")
    L = _lib()
    if scratch is None:
        need = L.endor_q4_scratch_bytes(m.rows, m.cols, m.group, nb)
        if need:
            scratch = torch.empty(need, dtype=torch.uint8, device=X.device)
    _on(m.packed.get_device(), X, Y, scratch)
    ldx = X.stride(0) if nb > 1 else m.cols
    _check(L.endor_q4_gemm(m.rows, m.cols, m.group, m.zeros, _dptr(m.packed), m.packed.numel(), _dtype_code(X.dtype), _dptr(X), ldx, nb,
                           _dptr(Y), _dptr(scratch), 0 if scratch is None else scratch.numel(), _stream_handle(stream)), "endor_q4_gemm")
    return Y
