"""Attention over sequences that are cut into parts: lengths alike and not, more sequences than a wave has lanes, wide heads that share, groups of more than
16 query heads with their weights, and a bound on the lengths far above them."""
import numpy as np
import pytest

from test_gpu_attn_decode import check, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("heads,dim", [((2, 1), 64), ((16, 1), 256), ((40, 2), 128), ((3, 3), 80)], ids=str)
def test_alike_and_not(heads, dim, dtype):
    print("attn parts", heads, dim, dtype, flush=True)
    for lengths in ([2500] * 3, [2500, 2100, 2400], [2500, 10, 0, 1300]):
        args = make(lengths, heads, dim, 64, dtype, seed=dim + len(lengths))
        check(*args, lengths, dtype)


@pytest.mark.parametrize("batch", [63, 64, 65, 130])
def test_many_sequences(batch):
    """The lengths of all sequences decide how each is cut, 64 at a time."""
    g = np.random.default_rng(batch)
    for lengths in (g.integers(1100, 1300, batch), np.where(g.random(batch) < 0.8, 3, 1200)):
        lengths = [int(n) for n in lengths]
        check(*make(lengths, (2, 2), 16, 64, torch.float16, seed=batch), lengths, torch.float16)


def test_weights_of_a_group_of_many_heads():
    for lengths in ([600, 33], [1500, 1400]):
        cache, q, k, v, table = make(lengths, (40, 1), 64, 32, torch.float16, seed=3)
        w = np.random.default_rng(4).random((2, 1, cache.capacity), dtype=np.float32)
        check(cache, q, k, v, table, lengths, torch.float16, weights=w, new_weights="same")


def test_bounds_far_above_the_lengths():
    """Most workgroups have no part."""
    lengths = [700, 5, 0]
    args = make(lengths, (4, 2), 64, 16, torch.bfloat16, seed=5, extra_pages=4000)
    assert args[0].capacity > 60000
    check(*args, lengths, torch.bfloat16)
    lengths = [130]
    check(*make(lengths, (8, 1), 128, 16, torch.float16, seed=6, extra_pages=4000), lengths, torch.float16)


def test_masks_over_parts():
    """Whole parts hidden, and a sequence hidden altogether, over sequences that are cut."""
    lengths = [3000, 3000, 2900]
    cache, q, k, v, table = make(lengths, (8, 2), 64, 16, torch.float16, seed=7)
    bits = np.random.default_rng(8).random((3, cache.capacity)) < 0.3
    bits[0, 200:2000] = False
    bits[1] = False
    mask = np.packbits(np.pad(bits, ((0, 0), (0, -cache.capacity % 64))), axis=1, bitorder="little").view(np.uint64)
    check(cache, q, k, v, table, lengths, torch.float16, mask=mask)
