"""A cache whose pool holds no pages yet, whatever strides torch gives it."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("how", ["torch", "numpy", "slots first"])
def test_nothing_is_attended_to(how):
    k = {"torch": lambda: torch.empty((0, 2, 16, 64), dtype=torch.float16, device="cuda"),
         "numpy": lambda: torch.from_numpy(np.empty((0, 2, 16, 64), np.float16)).cuda(),  # strides of 0
         "slots first": lambda: torch.empty((0, 16, 2, 64), dtype=torch.float16, device="cuda").transpose(1, 2)}[how]()
    cache = endor.KVCache(k, torch.empty((0, 2, 16, 64), dtype=torch.float16, device="cuda"), torch.full((3, 4), 9, dtype=torch.int32, device="cuda"))
    out, lse = endor.attn_decode(cache, torch.ones((3, 4, 64), dtype=torch.float16, device="cuda"), torch.full((3,), 60, dtype=torch.int32, device="cuda"))
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))
    new = torch.ones((3, 2, 64), dtype=torch.float16, device="cuda")
    n, _ = endor.kv_append(cache, new, new, torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert n.tolist() == [1, 1, 1]  # its slots are on pages that are not there
