"""Bounds that 32 bits do not hold keep their meaning.  No GPU needed: tensors lie in host memory, and the library is a recorder."""
import ctypes

import pytest

from paper_2406_11674_amd import decode
from test_decode_wide_groups import library  # noqa: F401  (a fixture)

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("wide", [1 << 31, 1 << 32, (1 << 32) + 5, 10 ** 12])
def test_bounds(library, wide):
    i32 = torch.int32
    pool, lengths = torch.zeros((4, 2, 16, 64), dtype=torch.float16), torch.zeros(2, dtype=i32)
    cache = decode.KVCache(pool, pool.clone(), torch.zeros((2, 2), dtype=i32))
    weights, positions = torch.zeros((2, 2, 32)), torch.zeros((2, 2, 32), dtype=i32)

    def passed(name, at):
        return [ctypes.c_int32(args[at]).value for n, args in library.calls if n == name]

    decode.attn_decode(cache, torch.zeros((2, 4, 64), dtype=torch.float16), lengths, max_len=wide)
    decode.kv_evict(cache, lengths, lengths, weights, positions, wide, 2, max_len=wide)
    decode.kv_evict(cache, lengths, lengths, weights, positions, 8, wide, max_len=-wide)
    assert passed("endor_attn_scratch_bytes", 2)[0] >= 32 and passed("endor_attn_decode", 6)[0] >= 32
    (budget, eight), (two, recent), (most, none) = (passed("endor_kv_evict", at) for at in (1, 2, 3))
    assert budget >= 32 and eight == 8 and two == 2 and recent > 8 and most >= 32 and none < 0  # a window wider than the budget is refused, and so is a bound below 0
    (first, second), (bound, below) = (passed("endor_kv_evict_scratch_bytes", at) for at in (1, 2))
    assert first >= 32 and second == 8 and bound >= 32 and below < 0
