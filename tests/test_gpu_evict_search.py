"""Eviction from rows whose weights lie close together on both sides of a bin's end, with zeros and a few far ones beside them: once a bin has given its
own ends, the next bins reach past them, where keys lie that have been counted already.  Bit for bit against the definition."""
import numpy as np
import pytest

from test_gpu_kv_cache import make, run_evict

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def below_one(g, n, ones):
    """Zeros, a cluster that ends with the number below one, and ones."""
    w = (0.98437488 + g.random(n) * (0.99999994 - 0.98437488)).astype(np.float32)
    w[:n // 8] = 0
    w[n // 8:n // 8 + 3] = np.float32([0.98437488, 0.99999994, 0.99999988])
    w[n // 8 + 3:n // 8 + 3 + ones] = 1
    return g.permutation(w)


def around_one(g, n):
    w = (0.9 + 0.2 * g.random(n)).astype(np.float32)
    return np.where(g.random(n) < 0.2, np.float32(0), w)


@pytest.mark.parametrize("length", [1708, 3500, 5000, 9000, 40000])
def test_clusters_across_the_ends_of_bins(length):
    print("evict clusters", length, flush=True)
    lengths = np.array([length] * 2, np.int32)
    cache, k, v, table, g = make(lengths, lengths, 4, 8, 64, seed=length)
    w = np.zeros((2, 4, cache.capacity), np.float32)
    for h, ones in enumerate((1, 5, 65, 400)):
        w[0, h, :length] = below_one(g, length, ones)
        w[1, h, :length] = around_one(g, length)
    pos = np.broadcast_to(np.arange(cache.capacity, dtype=np.int32), w.shape).copy()
    seen = np.full(2, 1 << 20, np.int32)  # no token is among the newest
    for budget in (2, 6, 64, 66, 401, length // 2, length - length // 8 - 1, length - 20, length - 1):
        run_evict(lengths, seen, w, pos, budget, 0, cache, k, v, table, in_place=budget % 2 == 0)
