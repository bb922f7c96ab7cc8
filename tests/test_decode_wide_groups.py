"""A group that 32 bits do not hold is refused: its scales would be counted by one number and read or written by another.  No GPU needed: tensors lie in host
memory, and the library is a recorder."""

import pytest

from paper_2406_11674_amd import decode

torch = pytest.importorskip("torch")


class Recorder:
    """Stands for the library: notes the arguments as the entry points get them, scratch sizes as they are asked for."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            return 256 if name.endswith("_bytes") else 0
        return entry


@pytest.fixture
def library(monkeypatch):
    recorder = Recorder()
    decode._torch()
    monkeypatch.setattr(decode, "_current_gpu", lambda: -1)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(decode, "_lib", lambda: recorder)
    return recorder


@pytest.mark.parametrize("group", [(1 << 32) + 32, (1 << 32) + 128, 1 << 40, -1, -(1 << 32) + 64])
def test_groups(library, group):
    dense = torch.zeros((16, 1000), dtype=torch.float16)
    with pytest.raises(ValueError):
        decode.q4_quantize(dense, group)
    codes, scales = torch.zeros((16, 500), dtype=torch.uint8), torch.zeros((16, 1), dtype=torch.float16)
    with pytest.raises(ValueError):
        decode.q4_pack(codes, scales, None, 1000, group)
    assert library.calls == []
