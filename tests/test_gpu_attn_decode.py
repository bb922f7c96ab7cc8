"""Attention of one new token over a paged cache against the definition in 64 bits: lengths around tiles, pages and splits,
shared heads, widths, masks, pages that are not there, strides, streams.  Everything that is not visible holds NaN or infinity.

Bounds, from the arithmetic (u = 2^-24).  A logit is a sum of at most 256 exact products in fp32, at most two roundings per instruction of
32 of them and one for the scale, and the exponent takes it relative to the maximum: off by d = (2 * dim / 32 + 8) u S, S the largest
scale * sum |q k|.  Weights p are then off by 2 d relative, their sum and the sums over v by at most 2 roundings per 32 slots
and 64 for joins; p enters the second product in two parts of the cache's type, which leaves 2^-16 of it in bfloat16 and
2^-20 in float16; the output is rounded once."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from oracle import decode_oracle as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24


def make(lengths, heads, dim, page, dtype, seed=0, spare=2, extra_pages=0, order="hpsd", steep=2.0):
    """A cache whose sequences hold their pages at random places; what no sequence holds is NaN and infinity."""
    g = np.random.default_rng(seed)
    q_heads, kv = heads
    need = [-(-n // page) for n in lengths]
    most = max(1, max(need) + extra_pages)
    count = sum(need) + spare
    perm = g.permutation(count)
    table = np.full((len(lengths), most), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b]) + n]
    k = torch.full((count, kv, page, dim), float("nan"))
    v = torch.full((count, kv, page, dim), float("inf"))
    for b, n in enumerate(lengths):
        for i in range(need[b]):
            m = min(page, n - i * page)
            k[table[b, i], :, :m] = torch.from_numpy(g.standard_normal((kv, m, dim), dtype=np.float32))
            v[table[b, i], :, :m] = torch.from_numpy(g.standard_normal((kv, m, dim), dtype=np.float32))
    k, v = k.to(dtype), v.to(dtype)
    q = (steep * torch.from_numpy(g.standard_normal((len(lengths), q_heads, dim), dtype=np.float32))).to(dtype)
    if order == "psh":  # [pages, page_size, heads, dim] in memory
        kd, vd = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (k, v))
    elif order == "pair":  # keys and values of a page side by side, room behind every slot
        both = torch.full((count, 2, kv, page, -(-dim // 8) * 8 + 8), float("nan"), dtype=dtype)
        both[:, 0, ..., :dim], both[:, 1, ..., :dim] = k, v
        both = both.cuda()
        kd, vd = both[:, 0, ..., :dim], both[:, 1, ..., :dim]
    else:
        kd, vd = k.cuda(), v.cuda()
    cache = endor.KVCache(kd, vd, torch.from_numpy(table).cuda())
    return cache, q, k.float().numpy(), v.float().numpy(), table


def check(cache, q, k, v, table, lengths, dtype, max_len=None, mask=None, scale=None, weights=None, new_weights="fresh", qd=None, out=None):
    dim, batch, q_heads = q.shape[2], q.shape[0], q.shape[1]
    most = cache.capacity if max_len is None else max_len
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    md = None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda()
    wd = None if weights is None else torch.from_numpy(weights).cuda()
    nd = None
    if new_weights == "fresh":
        nd = torch.full((batch, cache.kv_heads, cache.capacity), -7.0, device="cuda")
    elif new_weights == "same":
        nd = wd
    got, lse = endor.attn_decode(cache, q.cuda() if qd is None else qd, lens, max_len=max_len, mask=md, scale=scale, weights=wd, new_weights=nd, out=out)
    torch.cuda.synchronize()
    sc = dim ** -0.5 if scale is None else scale
    ref, rlse, probs, spread, steep = orc.attention(k, v, table, q.float().numpy(), lengths, most, sc, None if mask is None else mask)
    n = max([1] + [len(p[0]) for p in probs])
    d = (2 * dim / 32 + 8) * U * steep
    sums = (2 * n / 32 + 64) * U
    parts, half = (2.0 ** -16, 2.0 ** -8) if dtype == torch.bfloat16 else (2.0 ** -20, 2.0 ** -11)
    assert np.all(np.isfinite(got.float().cpu().numpy()))
    off = np.abs(got.float().cpu().numpy().astype(np.float64) - ref)
    assert np.all(off <= half * np.abs(ref) * 1.01 + (2 * d[..., None] + 2 * sums + parts) * spread + 2.0 ** -25), off.max()
    mine = lse.cpu().numpy().astype(np.float64)
    empty = np.isneginf(rlse)
    assert np.array_equal(empty, np.isneginf(mine))
    assert np.all(np.abs(mine[~empty] - rlse[~empty]) <= (d + sums + 4 * U * np.abs(rlse))[~empty])
    if nd is not None:
        w = nd.cpu().numpy().astype(np.float64)
        group = q_heads // cache.kv_heads
        for b in range(batch):
            length = max(0, min(lengths[b], most, cache.capacity))
            want = np.zeros((cache.kv_heads, length)) if weights is None else weights[b, :, :length].astype(np.float64)
            slots, p = probs[b]
            err = 2 * U * np.abs(want)
            for h in range(q_heads):
                want[h // group, slots] += p[h]
                err[h // group, slots] += p[h] * (2 * d[b, h] + sums + (4 + 2 * abs(rlse[b, h]) + group) * U) + U * want[h // group, slots]
            assert np.all(np.abs(w[b, :, :length] - want) <= err + 2 * U * np.abs(want) + 1e-37), np.abs(w[b, :, :length] - want).max()
            if new_weights == "fresh":
                assert np.all(w[b, :, length:] == -7.0)


LENGTHS = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (8, 2), (7, 1), (16, 1), (17, 1), (48, 2)], ids=str)
def test_lengths_around_tiles(heads, dtype):
    print("attn", heads, dtype, flush=True)
    for dim, page in ((64, 16), (128, 8)):
        args = make(LENGTHS, heads, dim, page, dtype, seed=dim + heads[0])
        check(*args, LENGTHS, dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 96, 120, 128, 136, 160, 192, 200, 256])
def test_widths(dim, dtype):
    print("attn dim", dim, dtype, flush=True)
    lengths = [0, 1, 33, 257, 100]
    check(*make(lengths, (10, 2), dim, 32, dtype, seed=dim), lengths, dtype)


@pytest.mark.parametrize("page", [8, 16, 32, 64, 256, 1024])
def test_pages_and_long_sequences(page):
    print("attn page", page, flush=True)
    lengths = [511, 512, 513, 1023, 1025, 2049, 4097, 5000, 3]
    check(*make(lengths, (4, 2), 64, page, torch.float16, seed=page), lengths, torch.float16)


def test_one_long_sequence():
    lengths = [40001]
    check(*make(lengths, (8, 1), 128, 64, torch.bfloat16, seed=1), lengths, torch.bfloat16)


@pytest.mark.parametrize("order", ["hpsd", "psh", "pair"])
def test_orders_and_strides_of_the_cache(order):
    lengths = [77, 0, 130]
    for dim in (64, 80):
        args = make(lengths, (6, 3), dim, 16, torch.float16, seed=3, order=order)
        check(*args, lengths, torch.float16)


def test_query_strides_and_alignment():
    """q as a slice of a projection's output, at every 2-byte alignment."""
    lengths = [50, 65]
    cache, q, k, v, table = make(lengths, (4, 2), 64, 16, torch.float16, seed=4)
    for off in (0, 1, 3, 8):
        buf = torch.full((2, 4 * 70 + 16), float("nan"), dtype=torch.float16, device="cuda")
        qd = torch.as_strided(buf, (2, 4, 64), (buf.stride(0), 70, 1), off)
        qd.copy_(q)
        check(cache, q, k, v, table, lengths, torch.float16, qd=qd)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_masks(dtype):
    """Random bits, whole tiles hidden, all hidden, left padding, one slot visible; hidden slots hold NaN and infinity."""
    g = np.random.default_rng(5)
    lengths = [200, 200, 200, 700, 64, 1]
    cache, q, k, v, table = make(lengths, (8, 2), 64, 16, dtype, seed=6)
    bits = g.random((6, 1024)) < 0.5
    bits[0, 32:128] = False
    bits[1] = False
    bits[2] = np.arange(1024) >= 150
    bits[3] = np.arange(1024) == 699
    bits[4] = True
    bits[5, 0] = False
    mask = np.packbits(bits, axis=1, bitorder="little").view(np.uint64)
    kd, vd = cache.k, cache.v
    for b, n in enumerate(lengths):
        for t in range(n):
            if not bits[b, t]:
                p = table[b, t // 16]
                kd[p, :, t % 16], vd[p, :, t % 16] = float("nan"), float("-inf")
                k[p, :, t % 16], v[p, :, t % 16] = np.nan, -np.inf
    check(cache, q, k, v, table, lengths, dtype, mask=mask)


def test_bounds_on_lengths_and_missing_pages():
    """Lengths below zero, past max_len and past the capacity; pages outside the pool in the middle of a sequence."""
    lengths = [100, 40, 90, 96]
    cache, q, k, v, table = make(lengths, (4, 4), 64, 16, torch.float16, seed=7)
    check(cache, q, k, v, table, [100, -5, 90, 1 << 30], torch.float16, max_len=50)
    table[0, 2], table[2, 0], table[3, 5] = -1, k.shape[0], 2 ** 31 - 1
    cache.pages.copy_(torch.from_numpy(table))
    check(cache, q, k, v, table, [100, 40, 90, 2 ** 31 - 1], torch.float16)


def test_no_slots_at_all():
    k = torch.zeros((0, 2, 16, 64), dtype=torch.float16, device="cuda")
    cache = endor.KVCache(k, k, torch.zeros((3, 0), dtype=torch.int32, device="cuda"))
    out, lse = endor.attn_decode(cache, torch.ones((3, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))
    cache = endor.KVCache(k, k, torch.full((3, 4), 9, dtype=torch.int32, device="cuda"))
    out, lse = endor.attn_decode(cache, torch.ones((3, 4, 64), dtype=torch.float16, device="cuda"), torch.full((3,), 60, dtype=torch.int32, device="cuda"))
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))


@pytest.mark.parametrize("how", ["fresh", "same"])
def test_accumulated_weights(how):
    lengths = [0, 1, 65, 513, 1100]
    cache, q, k, v, table = make(lengths, (16, 2), 64, 16, torch.float16, seed=8)
    w = np.random.default_rng(9).random((5, 2, cache.capacity), dtype=np.float32)
    check(cache, q, k, v, table, lengths, torch.float16, weights=w, new_weights=how)


def test_steep_logits():
    """Logits of hundreds: one slot takes all, the exponentials of the others underflow."""
    lengths = [300, 1000]
    check(*make(lengths, (4, 1), 128, 16, torch.float16, seed=10, steep=60.0), lengths, torch.float16)
    lengths = [300, 1000]
    args = make(lengths, (4, 1), 128, 16, torch.float16, seed=11)
    check(*args, lengths, torch.float16, scale=0.0)
    check(*args, lengths, torch.float16, scale=-0.3)


def test_values_of_all_sizes():
    """Keys that are subnormal, values up to the type's largest and down to its subnormals."""
    lengths = [100]
    cache, q, k, v, table = make(lengths, (2, 2), 64, 16, torch.float16, seed=12)
    for b in range(7):
        p = table[0, b]
        scale = (1.0, 2.0 ** -20, 1000.0, 2.0 ** -24, 0.0, 15000.0, 2.0 ** -14)[b]
        n = min(16, 100 - 16 * b)
        vv = (torch.from_numpy(v[p, :, :n]) * scale).half()
        cache.v[p, :, :n] = vv.cuda()
        v[p, :, :n] = vv.float().numpy()
    check(cache, q, k, v, table, lengths, torch.float16)


def test_offsets_past_32_bits():
    """Pages whose elements lie past 2^32 elements from the start of the pool."""
    page, dim, kv = 16, 64, 1
    far = (1 << 32) // 4 + 64  # elements between pages: page 5 begins past 2^32
    buf = torch.empty(5 * far + 2 * page * dim, dtype=torch.float16, device="cuda")
    kd = torch.as_strided(buf, (6, kv, page, dim), (far, page * dim, dim, 1), 0)
    vd = torch.as_strided(buf, (6, kv, page, dim), (far, page * dim, dim, 1), page * dim)
    g = np.random.default_rng(13)
    k, v = (torch.from_numpy(g.standard_normal((6, kv, page, dim), dtype=np.float32)).half() for _ in range(2))
    kd.copy_(k)
    vd.copy_(v)
    table = np.array([[5, 0, 4, 5]], np.int32)
    q = torch.from_numpy(g.standard_normal((1, 3, dim), dtype=np.float32)).half()
    check(endor.KVCache(kd, vd, torch.from_numpy(table).cuda()), q, k.float().numpy(), v.float().numpy(), table, [60], torch.float16)


def test_refusals():
    lengths = [20]
    cache, q, *_ = make(lengths, (4, 2), 64, 16, torch.float16)
    qd, lens = q.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    w = torch.zeros((1, 2, cache.capacity), device="cuda")
    for bad in (dict(q=qd.float()), dict(q=qd[:, :, :32]), dict(q=qd.cpu()), dict(lengths=lens.long()), dict(lengths=lens.cpu()),
                dict(mask=torch.zeros((1, 0), dtype=torch.int64, device="cuda")), dict(weights=w), dict(new_weights=w[..., :-1]),
                dict(out=torch.empty((1, 4, 64), device="cuda")), dict(lse=torch.empty((1, 4), dtype=torch.float16, device="cuda"))):
        with pytest.raises(ValueError):
            endor.attn_decode(**{"cache": cache, "q": qd, "lengths": lens, **bad})
    with pytest.raises(endor.EndorError):
        endor.attn_decode(cache, qd[:, :3], lens)  # three heads over two
    with pytest.raises(endor.EndorError):
        endor.attn_decode(cache, qd, lens, max_len=-1)
    k = cache.k
    with pytest.raises(ValueError):
        endor.KVCache(k, k[:, :1], cache.pages)
    with pytest.raises(ValueError):
        endor.KVCache(k.cpu(), k.cpu(), cache.pages.cpu())
    with pytest.raises(ValueError):
        endor.KVCache(k.float(), k.float(), cache.pages)
    with pytest.raises(ValueError):
        endor.KVCache(k, k, cache.pages.long())
    odd = torch.zeros((3, 2, 12, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(endor.EndorError):  # a page of 12 slots
        endor.attn_decode(endor.KVCache(odd, odd, cache.pages), qd, lens)
