"""Appends whose lengths and numbers of tokens seen share arrays: the answer depends neither on which ones nor on how many tokens come."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from oracle import decode_oracle as orc
from test_gpu_kv_cache import bits, ints, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("counted", [False, True], ids=["all", "counts"])
@pytest.mark.parametrize("outputs", ["none", "lengths", "seen", "both", "both in one"])
@pytest.mark.parametrize("tokens", [1, 8, 9, 40, 100])
def test_seen_defaults_to_the_lengths(tokens, outputs, counted):
    print("append", tokens, outputs, counted, flush=True)
    lengths = np.array([0, 1, 37, 130, 200], np.int32)  # the last two reach the capacity, or are past it
    cache, k, v, table, g = make(lengths, [144] * 5, 2, 64, 16, seed=tokens)
    cap = cache.capacity
    w, pos = g.random((5, 2, cap), dtype=np.float32), g.integers(0, 99, (5, 2, cap), dtype=np.int32)
    new = g.integers(-2 ** 15, 2 ** 15, (2, 5, tokens, 2, 64), dtype=np.int16)
    newd = torch.from_numpy(new).view(torch.float16).cuda()
    wd, pd, ld = torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda(), ints(lengths)
    counts = [tokens, 0, 5, tokens, 1] if counted else None
    kw = {"none": {}, "lengths": {"new_lengths": ld}, "seen": {"new_seen": ld}, "both": {"new_lengths": ld, "new_seen": torch.empty_like(ld)},
          "both in one": {"new_lengths": ld, "new_seen": ld}}[outputs]
    if outputs == "both in one":  # which can only be where both become the same
        lengths = lengths[:4]
        cache = endor.KVCache(cache.k, cache.v, cache.pages[:4])
        ld, wd, pd, newd, new, w, pos, table = ld[:4], wd[:4], pd[:4], newd[:, :4], new[:, :4], w[:4], pos[:4], table[:4]
        counts = counts and counts[:4]
        kw = {"new_lengths": ld, "new_seen": ld}
    n, s = endor.kv_append(cache, newd[0], newd[1], ld, counts=None if counts is None else ints(counts), weights=wd, positions=pd, **kw)
    torch.cuda.synchronize()
    want_n, want_s = orc.append(k, v, table, lengths, lengths, new[0], new[1], counts, w, pos)
    assert np.array_equal(n.cpu().numpy(), want_n) and np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(bits(cache.k), k) and np.array_equal(bits(cache.v), v)
    assert np.array_equal(wd.cpu().numpy(), w) and np.array_equal(pd.cpu().numpy(), pos)
    if "new_lengths" not in kw and "new_seen" not in kw:
        assert np.array_equal(ld.cpu().numpy(), lengths)
