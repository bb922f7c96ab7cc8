"""The decode side's entry points find wrong arguments on the host, before anything is launched."""
import ctypes

import paper_2406_11674_amd as endor
from paper_2406_11674_amd import decode

FAKE = 0x10000  # never dereferenced: every call below fails validation first, or has nothing to do


def cache(**kw):
    c = decode._Cache()
    c.d_k = c.d_v = c.d_pages = FAKE
    c.page_stride, c.head_stride, c.slot_stride, c.num_pages, c.pages_stride = 4096, 1024, 64, 10, 4
    c.batch, c.kv_heads, c.head_dim, c.page_size, c.max_pages, c.dtype = 2, 2, 64, 16, 4, 0
    for name, value in kw.items():
        setattr(c, name, value)
    return c


BAD_CACHES = [(dict(batch=-1), 1), (dict(kv_heads=0), 1), (dict(head_dim=0), 3), (dict(head_dim=60), 3), (dict(head_dim=264), 3),
              (dict(page_size=4), 3), (dict(page_size=24), 3), (dict(page_size=1 << 16), 3), (dict(max_pages=-1), 1),
              (dict(max_pages=1 << 27), 3), (dict(dtype=2), 3), (dict(d_k=FAKE + 8), 1), (dict(d_v=None), 1), (dict(d_pages=None), 1),
              (dict(d_pages=FAKE + 2), 1), (dict(pages_stride=3), 1), (dict(slot_stride=56), 1), (dict(head_stride=1028), 1),
              (dict(page_stride=-4096), 1), (dict(num_pages=-1), 1), (dict(num_pages=1 << 31), 1), (dict(batch=70000), 3)]


def append(c, k=FAKE, v=FAKE, strides=(128, 128, 64), tokens=1, counts=None, lengths=FAKE, seen=FAKE, lo=FAKE, so=FAKE, w=None, pos=None):
    return decode._lib().endor_kv_append(ctypes.addressof(c) if c else None, k, v, *strides, tokens, counts, lengths, seen, lo, so, w, pos, None)


def attend(c, heads=4, q=FAKE, qs=(256, 64), lengths=FAKE, max_len=64, mask=None, ms=0, out=FAKE, lse=None, w=None, wo=None, scratch=FAKE, size=1 << 30):
    return decode._lib().endor_attn_decode(ctypes.addressof(c) if c else None, heads, q, *qs, lengths, max_len, mask, ms, 1.0, out, lse, w, wo, scratch,
                                           size, None)


def evict(c, budget=8, recent=2, max_len=64, lengths=FAKE, seen=FAKE, w=FAKE, pos=FAKE, lo=FAKE, wo=FAKE, po=FAKE, scratch=FAKE, size=1 << 30):
    return decode._lib().endor_kv_evict(ctypes.addressof(c) if c else None, budget, recent, max_len, lengths, seen, w, pos, lo, wo, po, scratch, size, None)


def test_caches():
    for kw, status in BAD_CACHES:
        for call in (append, attend, evict):
            assert call(cache(**kw)) == status, (kw, call.__name__)
    for call in (append, attend, evict):
        assert call(None) == 1
        assert call(cache(batch=0)) == 0  # nothing to do


def test_append():
    for kw in (dict(k=None), dict(v=FAKE + 1), dict(strides=(-1, 0, 0)), dict(tokens=-1), dict(counts=FAKE + 2), dict(lengths=None), dict(seen=None),
               dict(lo=FAKE + 1), dict(so=None), dict(w=FAKE + 1), dict(pos=FAKE + 3)):
        assert append(cache(), **kw) == 1, kw


def test_attention():
    for kw in (dict(heads=0), dict(heads=3), dict(q=None), dict(q=FAKE + 1), dict(qs=(-1, 64)), dict(lengths=None), dict(max_len=-1), dict(mask=FAKE + 4, ms=9),
               dict(mask=FAKE, ms=0), dict(out=None), dict(out=FAKE + 1), dict(lse=FAKE + 2), dict(w=FAKE), dict(wo=FAKE + 2)):
        assert attend(cache(), **kw) == 1, kw
    big = cache(max_pages=1 << 12, pages_stride=1 << 12)
    need = decode._lib().endor_attn_scratch_bytes(ctypes.addressof(big), 4, 1 << 16, 1)
    assert need > 0 and need % 256 == 0
    assert attend(big, max_len=1 << 16, wo=FAKE, size=need - 1) == 2
    assert attend(big, max_len=1 << 16, wo=FAKE, scratch=FAKE + 16) == 1
    assert attend(big, max_len=1 << 16, wo=FAKE, scratch=None) == 1
    wrong, right = cache(dtype=5), cache()
    assert decode._lib().endor_attn_scratch_bytes(ctypes.addressof(wrong), 4, 64, 1) == 0
    assert decode._lib().endor_attn_scratch_bytes(ctypes.addressof(right), 3, 64, 1) == 0


def test_eviction():
    for kw in (dict(budget=-1, recent=0), dict(recent=9), dict(recent=-1), dict(max_len=-1), dict(lengths=None), dict(seen=FAKE + 2), dict(w=None), dict(pos=None),
               dict(lo=None), dict(wo=FAKE + 1), dict(po=None)):
        assert evict(cache(), **kw) == 1, kw
    c = cache()
    need = decode._lib().endor_kv_evict_scratch_bytes(ctypes.addressof(c), 8, 64)
    assert need > 0 and evict(cache(), size=need - 1) == 2 and evict(cache(), scratch=FAKE + 8) == 1
    assert decode._lib().endor_kv_evict_scratch_bytes(ctypes.addressof(c), -1, 64) == 0


def test_q4():
    L = decode._lib()
    assert L.endor_q4_bytes(16, 128, 128, 0) == 1024 + 256 and L.endor_q4_bytes(16, 128, 32, 1) == 1024 + 256
    for rows, cols, group in ((-1, 8, 32), (8, -1, 32), (8, 8, 16), (8, 8, 48), (8, 8, 1 << 16), (1 << 20, 1 << 20, 32), (1 << 26, 1, 32)):
        assert L.endor_q4_bytes(rows, cols, group, 0) == 0
    size = L.endor_q4_bytes(16, 128, 32, 0)

    def gemm(rows=16, cols=128, group=32, zeros=0, packed=FAKE, nbytes=size, dtype=0, x=FAKE, ldx=128, nb=2, y=FAKE, scratch=None, room=0):
        return L.endor_q4_gemm(rows, cols, group, zeros, packed, nbytes, dtype, x, ldx, nb, y, scratch, room, None)

    for kw, status in ((dict(rows=-1), 1), (dict(cols=-1), 1), (dict(nb=-1), 1), (dict(nb=17), 1), (dict(group=33), 3), (dict(dtype=2), 3), (dict(packed=None), 1),
                       (dict(packed=FAKE + 128), 1), (dict(nbytes=size - 1), 2), (dict(zeros=1, nbytes=0), 2), (dict(x=None), 1), (dict(x=FAKE + 1), 1),
                       (dict(ldx=127), 1), (dict(y=None), 1), (dict(y=FAKE + 2), 1), (dict(rows=1 << 20, cols=1 << 20), 3)):
        assert gemm(**kw) == status, kw
    assert gemm(rows=0) == 0 and gemm(nb=0) == 0
    wide = dict(rows=16, cols=100000, group=128, ldx=100000, nbytes=1 << 30)  # its columns are split, which takes scratch
    need = L.endor_q4_scratch_bytes(16, 100000, 128, 2)
    assert need > 0 and need % 256 == 0 and L.endor_q4_scratch_bytes(16, 128, 32, 2) == 0
    assert gemm(**wide) == 1 and gemm(scratch=FAKE + 8, room=need, **wide) == 1 and gemm(scratch=FAKE, room=need - 1, **wide) == 2
    for args in ((-1, 8, 32, 1), (16, 100000, 33, 1), (16, 100000, 128, 0), (16, 100000, 128, 17)):
        assert L.endor_q4_scratch_bytes(*args) == 0
    assert L.endor_q4_pack(16, 128, 32, None, FAKE, None, FAKE, size, None) == 1
    assert L.endor_q4_pack(16, 128, 32, FAKE, FAKE + 1, None, FAKE, size, None) == 1
    assert L.endor_q4_pack(16, 128, 32, FAKE, FAKE, None, FAKE + 8, size, None) == 1
    assert L.endor_q4_pack(16, 128, 32, FAKE, FAKE, None, FAKE, size - 1, None) == 2
    assert L.endor_q4_pack(16, 128, 40, FAKE, FAKE, None, FAKE, size, None) == 3
    assert L.endor_q4_pack(0, 128, 32, None, None, None, None, 0, None) == 0
    assert L.endor_q4_quantize(16, 128, 32, None, FAKE, FAKE, None, None) == 1
    assert L.endor_q4_quantize(16, 128, 32, FAKE, FAKE, FAKE + 1, None, None) == 1
    assert L.endor_q4_quantize(16, 128, 31, FAKE, FAKE, FAKE, None, None) == 3
    assert L.endor_q4_quantize(16, 0, 32, None, None, None, None, None) == 0


def test_names_are_public():
    for name in ("KVCache", "kv_append", "attn_decode", "kv_evict", "Q4Matrix", "q4_pack", "q4_quantize", "q4_gemm"):
        assert hasattr(endor, name)
