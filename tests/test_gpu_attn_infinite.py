"""Visible slots that hold infinities and NaN, at every head width: a slot whose logit is -infinity weighs nothing, whatever width its head has, and gives
bit for bit what hiding it gives; logits of +infinity and NaN, and values that are not finite, reach the outputs that they belong to and no others."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from test_gpu_attn_decode import check, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DIMS = [8, 16, 24, 40, 56, 64, 72, 96, 104, 120, 128, 136, 160, 200, 248, 256]


def attend(cache, q, lengths, mask=None):
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    w = torch.zeros((q.shape[0], cache.kv_heads, cache.capacity), device="cuda")
    md = None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda()
    out, lse = endor.attn_decode(cache, q.cuda(), lens, mask=md, new_weights=w)
    torch.cuda.synchronize()
    return out, lse, w


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", DIMS)
def test_keys_of_minus_infinity(dim, dtype):
    print("attn -inf", dim, dtype, flush=True)
    g = np.random.default_rng(dim)
    for lengths, heads in (([70, 33, 1], (6, 2)), ([3000, 40, 2500], (4, 1))):  # one launch, and parts
        cache, q, k, v, table = make(lengths, heads, dim, 16, dtype, seed=dim)
        q = q.abs() + 0.25  # so that such keys' logits are -infinity
        bits = np.ones((3, cache.capacity), bool)
        for b, n in enumerate(lengths):
            for i, t in enumerate(g.permutation(n)[:max(1, n // 9)]):
                at = int((0, 1, 7, dim - 1, dim // 2)[i % 5]) % dim
                cache.k[table[b, t // 16], :, t % 16, at] = float("-inf")
                bits[b, t] = False
        mask = np.packbits(np.pad(bits, ((0, 0), (0, -cache.capacity % 64))), axis=1, bitorder="little").view(np.uint64)
        seen, hidden = attend(cache, q, lengths), attend(cache, q, lengths, mask)
        for a, z in zip(seen, hidden):
            assert torch.equal(a, z)
        check(cache, q, k, v, table, lengths, dtype, mask=mask)


@pytest.mark.parametrize("dim", DIMS)
def test_what_is_not_finite_stays_with_its_own(dim):
    lengths = [200, 200, 200, 200]
    cache, q, k, v, table = make(lengths, (4, 2), dim, 16, torch.float16, seed=dim + 1)
    q = q.abs() + 0.25
    want = attend(cache, q, lengths)
    cache.k[table[1, 3], 1, 5, 0] = float("inf")
    cache.k[table[2, 0], 0, 15, dim - 1] = float("nan")
    cache.v[table[3, 12], 1, 7, dim // 2] = float("-inf")
    got = attend(cache, q, lengths)
    assert all(torch.isfinite(x[:, :, :200]).all() for x in (want[0], want[2])) and torch.isfinite(want[1]).all()
    broken = torch.zeros((4, 4, dim), dtype=torch.bool, device="cuda")
    broken[1, 2:] = broken[2, :2] = True
    broken[3, 2:, dim // 2] = True
    assert torch.equal(~torch.isfinite(got[0]), broken) and torch.equal(got[0][~broken], want[0][~broken])
    heads = broken.all(2) if dim > 1 else broken[..., 0]
    assert torch.equal(~torch.isfinite(got[1]), heads) and torch.equal(got[1][~heads], want[1][~heads])
    kv = heads.view(4, 2, 2).any(2)
    assert not torch.isfinite(got[2][kv][:, :200]).any() and torch.equal(got[2][~kv], want[2][~kv])
