"""Writes into the paged cache and eviction from it, bit for bit against the definition, ties, NaN and missing pages included."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from oracle import decode_oracle as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def make(lengths, room, heads, dim, page, dtype=torch.float16, seed=0, order="hpsd", gaps=False):
    """A pool of random bit patterns (their type never matters) with pages for `room` slots of every sequence."""
    g = np.random.default_rng(seed)
    need = [-(-n // page) for n in room]
    count = sum(need) + 2
    perm = g.permutation(count)
    table = np.full((len(lengths), max(1, max(need))), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b]) + n]
        if gaps and n > 2:
            table[b, 1] = (-1, count, 2 ** 31 - 1)[b % 3]
    k, v = (g.integers(-2 ** 15, 2 ** 15, (count, heads, page, dim), dtype=np.int16) for _ in range(2))
    kd, vd = torch.from_numpy(k).view(dtype), torch.from_numpy(v).view(dtype)
    if order == "psh":
        kd, vd = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (kd, vd))
    else:
        kd, vd = kd.cuda(), vd.cuda()
    return endor.KVCache(kd, vd, torch.from_numpy(table).cuda()), k, v, table, g


def bits(t):
    return t.contiguous().cpu().view(torch.int16).numpy()


def ints(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


@pytest.mark.parametrize("order", ["hpsd", "psh"])
@pytest.mark.parametrize("heads,dim,page", [(1, 8, 8), (2, 64, 16), (8, 128, 16), (3, 80, 32), (5, 256, 64), (72, 128, 16)])
def test_append_tokens(heads, dim, page, order):
    print("append", heads, dim, page, order, flush=True)
    lengths = np.array([0, 1, page - 1, page, 3 * page + 1], np.int32)
    for tokens, counts in ((1, None), (1, [1, 0, 1, -3, 7]), (page + 3, None), (2 * page + 5, [0, 1, page, 2 * page + 5, 10 ** 9])):
        cache, k, v, table, g = make(lengths, lengths + tokens, heads, dim, page, seed=tokens, order=order)
        cap = cache.capacity
        w, pos = g.random((5, heads, cap), dtype=np.float32), g.integers(0, 99, (5, heads, cap), dtype=np.int32)
        new = g.integers(-2 ** 15, 2 ** 15, (2, 5, tokens, heads, dim), dtype=np.int16)
        seen = lengths + np.int32(11)
        wd, pd = torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
        ld, sd = ints(lengths), ints(seen)
        newd = torch.from_numpy(new).view(torch.float16).cuda()
        counted = None if counts is None else ints(counts)
        a, z = endor.kv_append(cache, newd[0], newd[1], ld, sd, counts=counted, weights=wd, positions=pd)
        torch.cuda.synchronize()
        assert np.array_equal(ld.cpu().numpy(), lengths) and np.array_equal(sd.cpu().numpy(), seen)
        n, s = orc.append(k, v, table, lengths, seen, new[0], new[1], counts, w, pos)
        assert np.array_equal(bits(cache.k), k) and np.array_equal(bits(cache.v), v)
        assert np.array_equal(a.cpu().numpy(), n) and np.array_equal(z.cpu().numpy(), s)
        assert np.array_equal(wd.cpu().numpy(), w) and np.array_equal(pd.cpu().numpy(), pos)


def test_append_in_place_strided_unaligned_and_past_the_capacity():
    heads, dim, page = 3, 64, 16
    lengths = np.array([30, 47, 48, -4, 99], np.int32)  # the capacity is 48
    cache, k, v, table, g = make(lengths, [48] * 5, heads, dim, page, seed=2, gaps=True)
    assert cache.capacity == 48
    big = torch.from_numpy(g.integers(-2 ** 15, 2 ** 15, (5, 4, 2 * heads * 65 + 1), dtype=np.int16)).view(torch.float16).cuda()
    nk = torch.as_strided(big, (5, 4, heads, dim), (big.stride(0), big.stride(1), 65, 1), 1)
    nv = torch.as_strided(big, (5, 4, heads, dim), (big.stride(0), big.stride(1), 65, 1), 1 + heads * 65)
    ld, sd = ints(lengths), ints(lengths + 5)
    a, z = endor.kv_append(cache, nk, nv, ld, sd, new_lengths=ld, new_seen=sd)
    torch.cuda.synchronize()
    n, s = orc.append(k, v, table, lengths, lengths + 5, bits(nk), bits(nv))
    assert a is ld and z is sd and np.array_equal(ld.cpu().numpy(), n) and np.array_equal(sd.cpu().numpy(), s)
    assert np.array_equal(bits(cache.k), k) and np.array_equal(bits(cache.v), v)


def test_append_nothing():
    cache, k, v, table, g = make([3, 4], [16, 16], 2, 64, 16)
    ld = ints([3, 4])
    none = torch.zeros((2, 0, 2, 64), dtype=torch.float16, device="cuda")
    a, z = endor.kv_append(cache, none, none, ld)
    assert torch.equal(a, ld) and torch.equal(z, ld) and np.array_equal(bits(cache.k), k)
    empty = endor.KVCache(cache.k, cache.v, torch.zeros((2, 0), dtype=torch.int32, device="cuda"))
    a, _ = endor.kv_append(empty, none.new_ones((2, 3, 2, 64)), none.new_ones((2, 3, 2, 64)), ld)
    assert torch.all(a == 0) and np.array_equal(bits(cache.k), k)


def run_evict(lengths, seen, w, pos, budget, recent, cache, k, v, table, max_len=None, in_place=False):
    ld, sd, wd, pd = ints(lengths), ints(seen), torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
    kw = dict(new_lengths=ld, new_weights=wd, new_positions=pd) if in_place else dict(
        new_weights=torch.full_like(wd, -7.0), new_positions=torch.full_like(pd, -7))
    n, nw, npos = endor.kv_evict(cache, ld, sd, wd, pd, budget, recent, max_len=max_len, **kw)
    torch.cuda.synchronize()
    most = cache.capacity if max_len is None else max_len
    rw, rp = w.copy(), pos.copy()
    want = orc.evict(k, v, table, lengths, seen, rw, rp, budget, recent, most)
    assert np.array_equal(n.cpu().numpy(), want)
    assert np.array_equal(bits(cache.k), k) and np.array_equal(bits(cache.v), v)
    nw, npos = nw.cpu().numpy(), npos.cpu().numpy()
    for b in range(len(lengths)):
        m = want[b]
        assert np.array_equal(nw[b, :, :m].view(np.int32), rw[b, :, :m].view(np.int32)), b
        assert np.array_equal(npos[b, :, :m], rp[b, :, :m]), b
        if not in_place:
            assert np.all(nw[b, :, m:] == -7) and np.all(npos[b, :, m:] == -7)


def statistics(g, batch, heads, cap, kind):
    if kind == "ties":
        return g.integers(0, 4, (batch, heads, cap)).astype(np.float32)
    if kind == "equal":
        return np.full((batch, heads, cap), 0.25, np.float32)
    w = (-np.log1p(-g.random((batch, heads, cap)))).astype(np.float32) ** 3
    if kind == "odd":  # NaN, infinities, both zeros, negative and subnormal numbers
        at = g.integers(0, 12, w.shape)
        for i, x in enumerate([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.0, 1e-40, -1e-40]):
            w[at == i] = x
    return w


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("budget,recent", [(0, 0), (1, 0), (1, 1), (16, 5), (63, 63), (64, 0), (100, 20), (1000, 300), (2047, 7)])
def test_evict(budget, recent, kind):
    print("evict", budget, recent, kind, flush=True)
    lengths = np.array([0, 1, budget, budget + 1, budget + 17, 2 * budget + 3, 2100], np.int32)
    heads = 2
    cache, k, v, table, g = make(lengths, lengths, heads, 64, 16, seed=budget)
    w = statistics(g, 7, heads, cache.capacity, kind)
    # a cache that was evicted from before: positions in any order, as many tokens seen again
    pos = np.stack([np.stack([g.permutation(2 * cache.capacity)[:cache.capacity] for _ in range(heads)]) for _ in range(7)]).astype(np.int32)
    seen = np.full(7, 2 * cache.capacity, np.int32)
    run_evict(lengths, seen, w, pos, budget, recent, cache, k, v, table)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_plain_order_in_place(in_place):
    """Positions as appends leave them; protected tokens are the newest."""
    lengths = np.array([300, 1500, 129], np.int32)
    cache, k, v, table, g = make(lengths, lengths, 4, 128, 16, seed=5, order="psh")
    w = statistics(g, 3, 4, cache.capacity, "random")
    pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
    run_evict(lengths, lengths.copy(), w, pos, 128, 32, cache, k, v, table, in_place=in_place)


def test_evict_more_protected_than_the_budget():
    lengths = np.array([200], np.int32)
    cache, k, v, table, g = make(lengths, lengths, 2, 64, 16, seed=6)
    w = statistics(g, 1, 2, cache.capacity, "random")
    pos = np.full(w.shape, 1000, np.int32)
    pos[0, 0, :40] = 0
    run_evict(lengths, np.array([1000], np.int32), w, pos, 50, 10, cache, k, v, table)


@pytest.mark.parametrize("length", [4095, 8193, 40000, 70001])
def test_evict_long(length):
    print("evict long", length, flush=True)
    lengths = np.array([length, length // 3], np.int32)
    cache, k, v, table, g = make(lengths, lengths, 1, 8, 64, seed=length)
    for kind in ("random", "ties"):
        w = statistics(g, 2, 1, cache.capacity, kind)
        pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
        run_evict(lengths, lengths.copy(), w, pos, length // 2, 100, cache, k, v, table)


@pytest.mark.parametrize("length", [700, 2100, 5000, 9000, 40000])
def test_evict_weights_close_together(length):
    """Nearly all weights in one bin of the first pass, among them many equal ones, with far smaller and larger ones beside them."""
    print("evict close", length, flush=True)
    lengths = np.array([length, length], np.int32)
    cache, k, v, table, g = make(lengths, lengths, 2, 8, 64, seed=length)
    w = (1 + g.integers(0, 3000, (2, 2, cache.capacity)) * 2.0 ** -23).astype(np.float32)
    w[:, :, ::7] = np.float32(1 + 1500 * 2.0 ** -23)
    w[:, :, 3::101], w[:, :, 5::103], w[:, :, 9::211] = 0, 1e-30, 3e30
    w[1, 1] = np.where(g.random(cache.capacity) < 0.8, 0, w[1, 1])
    pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
    for budget in (length // 5, length // 2, length - length // 8, length - 2, length - 1):
        run_evict(lengths, lengths.copy(), w, pos, budget, 10, cache, k, v, table)


@pytest.mark.parametrize("batch,heads,length", [(3, 72, 5000), (4, 72, 5000), (4, 72, 9001), (9, 30, 16384), (9, 30, 16385), (300, 1, 513)])
def test_evict_many_rows(batch, heads, length):
    """More rows than compute units, and fewer; with few moves and with many."""
    print("evict rows", batch, heads, length, flush=True)
    lengths = np.full(batch, length, np.int32)
    lengths[0], lengths[-1] = length // 2, 7
    cache, k, v, table, g = make(lengths, lengths, heads, 8, 64, seed=length)
    for kind, budget in (("random", length - 20), ("ties", length // 3)):
        w = statistics(g, batch, heads, cache.capacity, kind)
        pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
        run_evict(lengths, lengths.copy(), w, pos, budget, budget // 4, cache, k, v, table)


@pytest.mark.parametrize("budget", [360, 150])
def test_offsets_past_32_bits(budget):
    """Pages whose elements lie past 2^32 elements from the start of the pool: appended to, then evicted from."""
    page, dim, kv, length = 128, 64, 1, 371
    far = (1 << 32) // 4 + 64  # elements between pages: page 5 begins past 2^32
    buf = torch.empty(5 * far + 2 * page * dim, dtype=torch.float16, device="cuda")
    kd, vd = (torch.as_strided(buf, (6, kv, page, dim), (far, page * dim, dim, 1), at) for at in (0, page * dim))
    g = np.random.default_rng(17)
    k, v = (g.integers(-2 ** 15, 2 ** 15, (6, kv, page, dim), dtype=np.int16) for _ in range(2))
    kd.copy_(torch.from_numpy(k).view(torch.float16))
    vd.copy_(torch.from_numpy(v).view(torch.float16))
    table = np.array([[4, 0, 5]], np.int32)
    cache = endor.KVCache(kd, vd, torch.from_numpy(table).cuda())
    for tokens in (1, 8, 9):  # at the third page's end
        new = torch.from_numpy(g.integers(-2 ** 15, 2 ** 15, (2, 1, tokens, kv, dim), dtype=np.int16)).view(torch.float16)
        n, _ = endor.kv_append(cache, new[0].cuda(), new[1].cuda(), ints([length]))
        assert n.tolist() == [length + tokens]
        for pool, x in ((k, new[0]), (v, new[1])):
            pool[5, 0, length - 256:length - 256 + tokens] = bits(x)[0, :, 0]
        assert np.array_equal(bits(cache.k), k) and np.array_equal(bits(cache.v), v)
    w = statistics(g, 1, kv, cache.capacity, "random")
    pos = np.arange(cache.capacity, dtype=np.int32)[None, None].copy()
    run_evict(np.array([380], np.int32), np.array([380], np.int32), w, pos, budget, 20, cache, k, v, table)


def test_evict_bounds_and_missing_pages():
    lengths = np.array([-3, 100, 2 ** 31 - 1, 90], np.int32)
    cache, k, v, table, g = make(lengths, [16, 100, 112, 96], 2, 64, 16, seed=8, gaps=True)
    w = statistics(g, 4, 2, cache.capacity, "random")
    pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
    run_evict(lengths, np.array([0, 100, 112, -50], np.int32), w, pos, 40, 10, cache, k, v, table, max_len=95)
    run_evict(lengths, np.array([0, 100, 112, 2 ** 31 - 1], np.int32), w, pos, 40, 40, cache, k, v, table)


def test_refusals():
    cache, k, v, table, g = make([20], [20], 2, 64, 16)
    ld = ints([20])
    w, pos = torch.zeros((1, 2, 32), device="cuda"), torch.zeros((1, 2, 32), dtype=torch.int32, device="cuda")
    for bad in (dict(weights=w.half()), dict(positions=pos.float()), dict(weights=w[:, :1]), dict(lengths=ld.long()), dict(seen=ld.cpu()),
                dict(new_lengths=ld.float())):
        with pytest.raises(ValueError):
            endor.kv_evict(**{"cache": cache, "lengths": ld, "seen": ld, "weights": w, "positions": pos, "budget": 8, "recent": 2, **bad})
    for budget, recent in ((-1, 0), (4, 5), (4, -1)):
        with pytest.raises(endor.EndorError):
            endor.kv_evict(cache, ld, ld, w, pos, budget, recent, scratch=torch.empty(4096, dtype=torch.uint8, device="cuda"))
    with pytest.raises(endor.EndorError):  # scratch too small
        endor.kv_evict(cache, ld, ld, w, pos, 8, 2, scratch=torch.empty(0, dtype=torch.uint8, device="cuda"))
    new = torch.zeros((1, 2, 64), dtype=torch.float16, device="cuda")
    for bad in (dict(k=new.float()), dict(v=new[:, :1]), dict(counts=ld.long()), dict(weights=w.double()), dict(k=new.cpu())):
        with pytest.raises(ValueError):
            endor.kv_append(**{"cache": cache, "k": new, "v": new, "lengths": ld, **bad})
