"""A cache and a packed weight are handles on what they were made of: another tensor put in its place would not be what calls read, so it is refused.  No GPU
needed: the tensors lie in host memory."""
import copy
import pickle

import pytest

from paper_2406_11674_amd import decode

torch = pytest.importorskip("torch")


def test_a_cache_stays_as_it_was_made(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    pool = torch.zeros((4, 2, 16, 64), dtype=torch.float16)
    cache = decode.KVCache(pool, pool.clone(), torch.zeros((2, 2), dtype=torch.int32))
    for name, value in (("k", pool.clone()), ("v", pool.clone()), ("pages", torch.zeros((2, 8), dtype=torch.int32)), ("capacity", 128), ("batch", 1)):
        with pytest.raises(AttributeError):
            setattr(cache, name, value)
    cache.layer = 7  # a program's own note
    cache.pages.fill_(1)  # what the tensors hold may change
    assert cache.capacity == 32 and cache._c.d_pages == cache.pages.data_ptr()


def test_a_packed_weight_stays_as_it_was_made():
    m = decode.Q4Matrix(16, 128, 32, False, torch.zeros(1280, dtype=torch.uint8))
    for name, value in (("packed", torch.zeros(1280, dtype=torch.uint8)), ("rows", 32), ("group", 64)):
        with pytest.raises(AttributeError):
            setattr(m, name, value)
    m.name = "keys"
    assert m._packed[:2] == (m.packed.data_ptr(), 1280)


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda m: pickle.loads(pickle.dumps(m))], ids=["copy", "deepcopy", "pickle"])
def test_a_copy_goes_by_its_own_address(how):
    m = decode.Q4Matrix(16, 128, 32, False, torch.arange(1280).to(torch.uint8))
    other = how(m)
    assert (other.rows, other.cols, other.group, other.zeros) == (16, 128, 32, False) and torch.equal(other.packed, m.packed)
    assert other._packed == (other.packed.data_ptr(), 1280, -1)
