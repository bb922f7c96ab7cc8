"""A call whose tensors lie on another GPU than the current one runs there: the entry points launch on the current GPU, so the binding makes the tensors'
one current for the call.  No GPU needed: the tensors lie in host memory, whose number (-1) is not the current one's, and the library is a recorder."""
import contextlib

import pytest

from paper_2406_11674_amd import decode

torch = pytest.importorskip("torch")


class Recorder:
    """Stands for the library: notes which GPU is current when an entry point is called."""

    def __init__(self, current):
        self.current, self.calls = current, []

    def __getattr__(self, name):
        def entry(*args):
            if name.endswith("_bytes"):
                return 256
            self.calls.append((name, self.current[-1]))
            return 0
        return entry


@pytest.fixture(params=[0, -1], ids=["another is current", "theirs is current"])
def library(request, monkeypatch):
    current = [request.param]

    @contextlib.contextmanager
    def device(index):
        current.append(index)
        yield
        current.pop()

    recorder = Recorder(current)
    decode._torch()
    monkeypatch.setattr(decode, "_current_gpu", lambda: current[-1], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(decode, "_lib", lambda: recorder)
    return recorder


def test_every_call(library):
    i32 = torch.int32
    pool, lengths = torch.zeros((4, 2, 16, 64), dtype=torch.float16), torch.zeros(2, dtype=i32)
    cache = decode.KVCache(pool, pool.clone(), torch.zeros((2, 2), dtype=i32))
    new = torch.zeros((2, 2, 64), dtype=torch.float16)
    weights, positions = torch.zeros((2, 2, 32)), torch.zeros((2, 2, 32), dtype=i32)
    decode.kv_append(cache, new, new, lengths, weights=weights, positions=positions)
    decode.attn_decode(cache, new, lengths)
    decode.kv_evict(cache, lengths, lengths, weights, positions, 8, 2)
    codes, scales, _ = decode.q4_quantize(torch.zeros((16, 64), dtype=torch.float16), 32)
    m = decode.q4_pack(codes, scales, None, 64, 32)
    decode.q4_gemm(m, torch.zeros((2, 64), dtype=torch.float16))
    assert library.calls == [(name, -1) for name in ("endor_kv_append", "endor_attn_decode", "endor_kv_evict", "endor_q4_quantize", "endor_q4_pack",
                                                     "endor_q4_gemm")]
    assert len(library.current) == 1
