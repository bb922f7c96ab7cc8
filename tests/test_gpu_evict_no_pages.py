"""Eviction where the pool has no pages, or a sequence none of them: no key or value is looked for, weights and positions go by the definition."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from test_gpu_kv_cache import run_evict, statistics

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("count", [0, 1, 3])
@pytest.mark.parametrize("length,budget", [(40, 20), (129, 128), (2100, 2090), (2100, 1000), (40000, 39990), (40000, 100), (40000, 9000)])
def test_no_page_is_there(length, budget, count, in_place):
    """A pool of `count` pages of which the sequences have none: few moves, which the selecting workgroup does, and many."""
    print("evict without pages", length, budget, count, in_place, flush=True)
    g = np.random.default_rng(length + budget)
    k, v = (g.integers(-2 ** 15, 2 ** 15, (count, 2, 16, 64), dtype=np.int16) for _ in range(2))
    pages = -(-length // 16)
    table = np.where(g.random((2, pages)) < 0.5, -1, count).astype(np.int32)
    cache = endor.KVCache(*(torch.from_numpy(x).view(torch.float16).cuda() for x in (k, v)), torch.from_numpy(table).cuda())
    assert (cache.k.data_ptr() == 0) == (count == 0)
    lengths = np.array([length, budget - 3], np.int32)
    w = statistics(g, 2, 2, cache.capacity, "random")
    pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
    run_evict(lengths, lengths.copy(), w, pos, budget, budget // 4, cache, k, v, table, in_place=in_place)
