"""The decode side: a paged key-value cache with the attention that reads it, eviction from it, and products with
4-bit weights.  Argument marshalling over include/endor.h, as in `binding`; every step runs inside libendor.so."""
from __future__ import annotations

import contextlib
import ctypes
from dataclasses import dataclass

from . import binding
from .binding import _check, _dptr, _i64, _p, _sz

__all__ = ["KVCache", "kv_append", "attn_decode", "kv_evict", "Q4Matrix", "q4_pack", "q4_quantize", "q4_scratch_bytes", "q4_gemm"]

_i32 = ctypes.c_int32


class _Cache(ctypes.Structure):
    _fields_ = [("d_k", _p), ("d_v", _p), ("page_stride", _i64), ("head_stride", _i64), ("slot_stride", _i64),
                ("num_pages", _i64), ("d_pages", _p), ("pages_stride", _i64), ("batch", _i32), ("kv_heads", _i32),
                ("head_dim", _i32), ("page_size", _i32), ("max_pages", _i32), ("dtype", _i32)]


_lib_declared = None
_torch_module = None
_current_gpu = None


def _torch():
    global _torch_module, _current_gpu
    if _torch_module is None:
        import torch
        _torch_module = torch
        # not part of torch's interface: 0.1 us for 0.24
        _current_gpu = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _torch_module


def _lib():
    global _lib_declared
    L = binding._lib
    if L is None or _lib_declared is not L:
        L = binding.lib()
        for name, args in (
                ("endor_kv_append", [_p, _p, _p, _i64, _i64, _i64, ctypes.c_int, _p, _p, _p, _p, _p, _p, _p, _p]),
                ("endor_attn_decode", [_p, ctypes.c_int, _p, _i64, _i64, _p, _i32, _p, _i64, ctypes.c_float, _p, _p, _p, _p, _p, _sz, _p]),
                ("endor_kv_evict", [_p, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _p]),
                ("endor_q4_pack", [_i64, _i64, ctypes.c_int, _p, _p, _p, _p, _sz, _p]),
                ("endor_q4_quantize", [_i64, _i64, ctypes.c_int, _p, _p, _p, _p, _p]),
                ("endor_q4_gemm", [_i64, _i64, ctypes.c_int, ctypes.c_int, _p, _sz, ctypes.c_int, _p, _i64, ctypes.c_int, _p, _p, _sz, _p])):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = args
        for name, args in (("endor_attn_scratch_bytes", [_p, ctypes.c_int, _i32, ctypes.c_int]),
                           ("endor_kv_evict_scratch_bytes", [_p, _i32, _i32]),
                           ("endor_q4_bytes", [_i64, _i64, ctypes.c_int, ctypes.c_int]),
                           ("endor_q4_scratch_bytes", [_i64, _i64, ctypes.c_int, ctypes.c_int])):
            getattr(L, name).restype = _sz
            getattr(L, name).argtypes = args
        _lib_declared = L
    return L


def _stream(stream, device):
    """The handle of the stream that a call goes to: the given one, or the current one of the tensors' GPU."""
    if stream is not None:
        return stream.cuda_stream
    try:
        return _torch_module._C._cuda_getCurrentRawStream(device)  # not part of torch's interface: 0.2 us for 2.9
    except AttributeError:
        return int(_torch().cuda.current_stream(device).cuda_stream)


def _on(device, entry):
    """The library's entry point, called with that GPU as the current one."""
    def there(*args):
        with _torch().cuda.device(device):
            return entry(*args)
    return there


# The checks of a call are on the way of every token, and a tensor's attributes take 50 ns each: they are asked for
# once, tensor by tensor, and not through helpers (an append took 10 us of the host with those, the kernel 4).

def _of(stream):
    """What a call allocates, copies or clears for itself belongs to the stream that its kernels run on."""
    return contextlib.nullcontext() if stream is None else _torch().cuda.stream(stream)


def _bad(what):
    raise ValueError(what)


def _saturated(n):
    """A bound as the library gets it: 32 bits, and still above or below all that it is compared with."""
    return max(-1, min(n, 0x7fffffff))


def _dtype_code(dtype):
    torch = _torch()
    if dtype is torch.float16:
        return 0
    if dtype is torch.bfloat16:
        return 1
    raise ValueError("elements are float16 or bfloat16, got %s" % dtype)


class KVCache:
    """A paged cache: k and v are pools of pages [pages, kv_heads, page_size, head_dim] (any strides whose last is 1 and
    whose others are multiples of 8 elements; the same for both), `pages` the int32 table [batch, max_pages] of every
    sequence's pages.  The tensors stay the caller's: what they hold may change between calls, the tensors may not (another table of pages is
    another KVCache)."""

    def __init__(self, k, v, pages):
        torch = _torch()
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.device != pages.device:
            raise ValueError("k and v must be alike, [pages, kv_heads, page_size, head_dim], on the table's device")
        if pages.dtype != torch.int32 or pages.dim() != 2 or (pages.shape[1] > 1 and pages.stride(1) != 1):
            raise ValueError("pages must be an int32 tensor [batch, max_pages] with contiguous rows")
        empty = k.numel() == 0
        if not empty and (any(n > 1 and a != b for n, a, b in zip(k.shape, k.stride(), v.stride())) or (k.shape[3] > 1 and k.stride(3) != 1)):
            raise ValueError("k and v must have the same strides, the last one 1")
        if not k.is_cuda:
            raise ValueError("the cache lies in GPU memory")
        self.k, self.v, self.pages, self.device_index = k, v, pages, k.get_device()
        self.num_pages, self.kv_heads, self.page_size, self.head_dim = (int(n) for n in k.shape)
        self.batch, self.max_pages = int(pages.shape[0]), int(pages.shape[1])
        self.capacity = self.max_pages * self.page_size
        c = self._c = _Cache()
        c.d_k, c.d_v, c.d_pages = _dptr(k), _dptr(v), _dptr(pages)
        # the stride over a dimension of one element is never used, whatever torch says it is, and an empty pool's are not either
        c.page_stride, c.head_stride, c.slot_stride = (int(k.stride(i)) if k.shape[i] > 1 and not empty else -(-self.head_dim // 8) * 8 for i in range(3))
        c.num_pages, c.pages_stride = self.num_pages, int(pages.stride(0)) if self.batch > 1 else self.max_pages
        c.batch, c.kv_heads, c.head_dim, c.page_size, c.max_pages = self.batch, self.kv_heads, self.head_dim, self.page_size, self.max_pages
        c.dtype = _dtype_code(k.dtype)
        self.dtype = k.dtype
        self._at = ctypes.addressof(c)

    def __setattr__(self, name, value):
        if "_at" in self.__dict__ and name in self.__dict__:  # calls go by the addresses that were taken when it was made
            raise AttributeError("a KVCache stays as it was made: make another one for other tensors")
        object.__setattr__(self, name, value)

    def _scratch(self, nbytes):
        return _torch().empty(nbytes, dtype=_torch().uint8, device=self.k.device) if nbytes else None

    def attn_scratch(self, q_heads, max_len=None, weights=False):
        """Scratch of attn_decode for calls with these bounds; None if it takes none.  Calls that overlap in time need distinct ones."""
        return self._scratch(_lib().endor_attn_scratch_bytes(self._at, q_heads, self.capacity if max_len is None else _saturated(max_len), int(weights)))

    def evict_scratch(self, budget, max_len=None):
        """Scratch of kv_evict, likewise."""
        return self._scratch(_lib().endor_kv_evict_scratch_bytes(self._at, _saturated(budget), self.capacity if max_len is None else _saturated(max_len)))

    def _per_sequence(self, *tensors):
        i32, batch, device = _torch_module.int32, self.batch, self.device_index
        for t in tensors:
            if t.dtype is not i32 or t.get_device() != device or t.numel() != batch or not t.is_contiguous():
                _bad("lengths, seen, counts and what they become must be contiguous int32 tensors [batch] on the cache's GPU")

    def _per_slot(self, dtype, *tensors):
        shape, device = (self.batch, self.kv_heads, self.capacity), self.device_index
        for t in tensors:
            if t is not None and (t.dtype is not dtype or t.get_device() != device or t.shape != shape or not t.is_contiguous()):
                _bad("weights (float32) and positions (int32) must be contiguous tensors [batch, kv_heads, capacity] on the cache's GPU")

    def _take(self, scratch):
        if scratch is None:
            return None, 0
        if scratch.get_device() != self.device_index or not scratch.is_contiguous():
            _bad("scratch must be contiguous, on the cache's GPU")
        return scratch.data_ptr(), scratch.numel() * scratch.element_size()


def kv_append(cache, k, v, lengths, seen=None, counts=None, weights=None, positions=None, new_lengths=None, new_seen=None, stream=None):
    """endor_kv_append.  k, v: [batch, tokens, kv_heads, head_dim], or without `tokens` for one each.  `seen` defaults to
    `lengths` (nothing was evicted).  Returns (new_lengths, new_seen); pass lengths and seen for them to advance in place."""
    torch = _torch()
    if k.dim() == 3:
        k, v = k.unsqueeze(1), v.unsqueeze(1)
    shape, dtype, device = k.shape, cache.dtype, cache.device_index
    if len(shape) != 4 or v.shape != shape or k.dtype is not dtype or v.dtype is not dtype or k.get_device() != device or v.get_device() != device:
        _bad("k and v must be [batch, tokens, kv_heads, head_dim] of the cache's type, on its GPU")
    batch, tokens, heads, dim = shape
    if batch != cache.batch or heads != cache.kv_heads or dim != cache.head_dim:
        _bad("k and v must be [batch, tokens, kv_heads, head_dim] of the cache")
    st = k.stride()
    if v.stride() != st or st[3] != 1:
        with _of(stream):
            k, v = k.contiguous(), v.contiguous()
        st = k.stride()
    if seen is None:
        seen = lengths
    if new_lengths is None or new_seen is None:
        with _of(stream):
            new_lengths = torch.empty_like(lengths) if new_lengths is None else new_lengths
            new_seen = torch.empty_like(seen) if new_seen is None else new_seen
    cache._per_sequence(lengths, seen, new_lengths, new_seen)
    if counts is not None:
        cache._per_sequence(counts)
    if weights is not None:
        cache._per_slot(torch.float32, weights)
    if positions is not None:
        cache._per_slot(torch.int32, positions)
    entry = _lib().endor_kv_append
    if _current_gpu() != device:
        entry = _on(device, entry)
    status = entry(cache._at, k.data_ptr(), v.data_ptr(), st[0], st[1], st[2], tokens, None if counts is None else counts.data_ptr(),
                   lengths.data_ptr(), seen.data_ptr(), new_lengths.data_ptr(), new_seen.data_ptr(),
                   None if weights is None else weights.data_ptr(), None if positions is None else positions.data_ptr(), _stream(stream, device))
    if status:
        _check(status, "endor_kv_append")
    return new_lengths, new_seen


def attn_decode(cache, q, lengths, max_len=None, mask=None, scale=None, weights=None, new_weights=None, out=None, lse=None, scratch=None,
                stream=None):
    """endor_attn_decode.  q: [batch, q_heads, head_dim] of the cache's type; lengths: int32 [batch] on the device; max_len: the host's
    bound on them (default: the capacity); mask: int64 words [batch, >= ceil(max_len / 64)], a 0 bit hides its slot; scale defaults
    to head_dim ** -0.5.  With new_weights the tokens' attention weights are added to `weights` (None: to 0) into it.
    Returns (out, lse)."""
    torch = _torch()
    batch, device = cache.batch, cache.device_index
    max_len = cache.capacity if max_len is None else max_len if -1 <= max_len <= 0x7fffffff else _saturated(max_len)
    shape = q.shape
    if len(shape) != 3 or q.dtype is not cache.dtype or q.get_device() != device or shape[0] != batch or shape[2] != cache.head_dim:
        _bad("q must be [batch, q_heads, head_dim] of the cache's type, on its GPU")
    q_heads, st = shape[1], q.stride()
    if st[2] != 1:
        _bad("the last stride of q must be 1")
    cache._per_sequence(lengths)
    mask_at, mask_stride = None, 0
    if mask is not None:
        words = (min(max_len, cache.capacity) + 63) // 64
        if (mask.dtype is not torch.int64 or mask.dim() != 2 or mask.shape[0] != batch or mask.shape[1] < words or mask.get_device() != device
                or (mask.shape[1] > 1 and mask.stride(1) != 1)):
            _bad("mask must be an int64 tensor [batch, >= %d] with contiguous rows, on the cache's GPU" % words)
        mask_at, mask_stride = mask.data_ptr(), mask.stride(0) if batch > 1 else mask.shape[1]
    if weights is not None and new_weights is None:
        _bad("weights without new_weights: pass the buffer for the sums, which may be weights itself")
    if new_weights is not None:
        cache._per_slot(torch.float32, weights, new_weights)
    if out is None or lse is None or scratch is None:
        with _of(stream):
            if out is None:
                out = torch.empty((batch, q_heads, cache.head_dim), dtype=q.dtype, device=q.device)
            if lse is None:
                lse = torch.empty((batch, q_heads), dtype=torch.float32, device=q.device)
            if scratch is None:
                scratch = cache.attn_scratch(q_heads, max_len, new_weights is not None)
    if out.dtype is not cache.dtype or out.shape != shape or out.get_device() != device or not out.is_contiguous():
        _bad("out must be a contiguous tensor like q")
    if lse.dtype is not torch.float32 or lse.numel() != batch * q_heads or lse.get_device() != device or not lse.is_contiguous():
        _bad("lse must be a contiguous float32 tensor [batch, q_heads]")
    scratch_at, room = cache._take(scratch)
    entry = _lib().endor_attn_decode
    if _current_gpu() != device:
        entry = _on(device, entry)
    status = entry(cache._at, q_heads, q.data_ptr(), st[0], st[1], lengths.data_ptr(), max_len, mask_at, mask_stride,
                   cache.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), lse.data_ptr(),
                   None if weights is None else weights.data_ptr(), None if new_weights is None else new_weights.data_ptr(),
                   scratch_at, room, _stream(stream, device))
    if status:
        _check(status, "endor_attn_decode")
    return out, lse


def kv_evict(cache, lengths, seen, weights, positions, budget, recent, max_len=None, new_lengths=None, new_weights=None, new_positions=None,
             scratch=None, stream=None):
    """endor_kv_evict: every kv head of every sequence keeps `budget` tokens, the newest `recent` and those of the largest weight.
    Returns (new_lengths, new_weights, new_positions); pass the inputs for them to change in place."""
    torch = _torch()
    max_len = cache.capacity if max_len is None else max_len
    if not -1 <= max_len <= 0x7fffffff >= budget >= recent >= -1:
        budget, recent, max_len = _saturated(budget), _saturated(recent), _saturated(max_len)
    if new_lengths is None or new_weights is None or new_positions is None or scratch is None:
        with _of(stream):
            new_lengths = torch.empty_like(lengths) if new_lengths is None else new_lengths
            new_weights = torch.zeros_like(weights) if new_weights is None else new_weights
            new_positions = torch.zeros_like(positions) if new_positions is None else new_positions
            if scratch is None:
                scratch = cache.evict_scratch(budget, max_len)
    cache._per_sequence(lengths, seen, new_lengths)
    cache._per_slot(torch.float32, weights, new_weights)
    cache._per_slot(torch.int32, positions, new_positions)
    scratch_at, room = cache._take(scratch)
    device = cache.device_index
    entry = _lib().endor_kv_evict
    if _current_gpu() != device:
        entry = _on(device, entry)
    status = entry(cache._at, budget, recent, max_len, lengths.data_ptr(), seen.data_ptr(), weights.data_ptr(),
                   positions.data_ptr(), new_lengths.data_ptr(), new_weights.data_ptr(), new_positions.data_ptr(),
                   scratch_at, room, _stream(stream, device))
    if status:
        _check(status, "endor_kv_evict")
    return new_lengths, new_weights, new_positions


# ------------------------------------------------------------------ 4-bit weights

@dataclass
class Q4Matrix:
    """A 4-bit weight in the form the products read (device memory).  It stays as it was made: calls go by the address taken then."""
    rows: int
    cols: int
    group: int
    zeros: bool     # whether it has zero points of its own
    packed: object  # torch.uint8, the tensor of q4_pack

    def __post_init__(self):
        self._scratch = {}  # bytes by the number of right-hand sides: a plan's figures, asked for once
        self._packed = (self.packed.data_ptr(), self.packed.numel(), self.packed.get_device())

    def __setattr__(self, name, value):
        if "_packed" in self.__dict__ and name in self.__dict__:
            raise AttributeError("a Q4Matrix stays as it was made: make another one for another weight")
        object.__setattr__(self, name, value)

    def __reduce__(self):  # a copy goes by its own address
        return Q4Matrix, (self.rows, self.cols, self.group, self.zeros, self.packed)


def _q4_groups(cols, group):
    return -(-cols // group)


def q4_pack(codes, scales, zeros, cols, group, stream=None):
    """endor_q4_pack.  codes: uint8 [rows, (cols + 1) // 2], the even column in the low half; scales: float16 [rows, ceil(cols / group)];
    zeros: uint8 of that shape, or None for 8 everywhere.  Returns a Q4Matrix."""
    torch = _torch()
    if not 1 <= group <= 0x7fffffff:  # the library gets its low 32 bits, by which it counts the groups of a row
        raise ValueError("group must be a power of two from 32 to 32768")
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
    if any(t is not None and t.get_device() != codes.get_device() for t in (scales, zeros)):
        raise ValueError("codes, scales and zeros must be on one GPU")
    L = _lib()
    with _of(stream):
        packed = torch.empty(L.endor_q4_bytes(rows, cols, group, int(zeros is not None)), dtype=torch.uint8, device=codes.device)
    device = codes.get_device()
    entry = L.endor_q4_pack
    if _current_gpu() != device:
        entry = _on(device, entry)
    _check(entry(rows, cols, group, _dptr(codes), _dptr(scales), _dptr(zeros), _dptr(packed), packed.numel(), _stream(stream, device)),
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
    if not 1 <= group <= 0x7fffffff:  # the library gets its low 32 bits, by which it counts the groups of a row
        raise ValueError("group must be a power of two from 32 to 32768")
    with _of(stream):
        codes = torch.empty((rows, (cols + 1) // 2), dtype=torch.uint8, device=dense.device)
        scales = torch.empty((rows, _q4_groups(cols, group)), dtype=torch.float16, device=dense.device)
        points = torch.empty(scales.shape, dtype=torch.uint8, device=dense.device) if zeros else None
    device = dense.get_device()
    entry = _lib().endor_q4_quantize
    if _current_gpu() != device:
        entry = _on(device, entry)
    _check(entry(rows, cols, group, _dptr(dense), _dptr(codes), _dptr(scales), _dptr(points), _stream(stream, device)),
           "endor_q4_quantize")
    return codes, scales, points


def q4_scratch_bytes(m, nb):
    """endor_q4_scratch_bytes: scratch of q4_gemm with that many right-hand sides; mostly none."""
    need = m._scratch.get(nb)
    if need is None:
        need = m._scratch[nb] = int(_lib().endor_q4_scratch_bytes(m.rows, m.cols, m.group, nb))
    return need


def q4_gemm(m, X, Y=None, scratch=None, stream=None):
    """endor_q4_gemm: Y (fp32, nb x rows) = X W^T; X: (nb, cols) float16 or bfloat16 (row stride = ldx), nb <= 16."""
    torch, dtype = _torch(), X.dtype
    at, room, device = m._packed
    (nb, cols), (ldx, inner), rows = X.shape, X.stride(), m.rows  # a ValueError if X is not a matrix
    if cols != m.cols or X.get_device() != device or (inner != 1 and cols > 1):
        _bad("X must be (nb, cols) with contiguous rows, on the weight's GPU")
    if Y is None:
        with _of(stream):
            Y = torch.empty((nb, rows), dtype=torch.float32, device=X.device)
    elif Y.dtype is not torch.float32 or Y.numel() != nb * rows or Y.get_device() != device or not Y.is_contiguous():
        _bad("Y must be a contiguous fp32 tensor of nb*rows elements, on the weight's GPU")
    scratch_at, space = None, 0
    if scratch is None:
        need = q4_scratch_bytes(m, nb)
        if need:
            with _of(stream):
                scratch = torch.empty(need, dtype=torch.uint8, device=X.device)
    elif scratch.get_device() != device or not scratch.is_contiguous():
        _bad("scratch must be contiguous, on the weight's GPU")
    if scratch is not None:
        scratch_at, space = scratch.data_ptr(), scratch.numel() * scratch.element_size()
    entry = _lib().endor_q4_gemm
    if _current_gpu() != device:
        entry = _on(device, entry)
    status = entry(rows, cols, m.group, m.zeros, at, room, 0 if dtype is torch.float16 else _dtype_code(dtype), X.data_ptr(),
                   ldx if nb > 1 else cols, nb, Y.data_ptr(), scratch_at, space, _stream(stream, device))
    if status:
        _check(status, "endor_q4_gemm")
    return Y
