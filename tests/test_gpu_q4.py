"""Products with 4-bit weights against the definition in 64 bits.

Bound (u = 2^-24): a group's products (code - zero) * x are exact in fp32; an instruction that adds 32 of them to a sum is charged two roundings, scaling and
adding a group two more, and joining parts of a row at most 64: off by at most (cols / 16 + 2 * groups + 64) u sum |w x|."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from oracle import decode_oracle as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def make(rows, cols, group, zeros, seed=0):
    g = np.random.default_rng(seed)
    groups = -(-cols // group)
    codes = g.integers(0, 256, (rows, (cols + 1) // 2), dtype=np.uint8)  # an odd row's last half byte is rubbish
    scales = (0.001 + 0.01 * g.random((rows, groups))).astype(np.float16)
    z = g.integers(0, 16, (rows, groups), dtype=np.uint8) if zeros else None
    dev = [None if a is None else torch.from_numpy(a).cuda() for a in (codes, scales, z)]
    return endor.q4_pack(*dev, cols, group), orc.q4_dense(codes, scales, z, cols, group), g


def check(m, w, x, dev=None, **kw):
    y = endor.q4_gemm(m, x.cuda() if dev is None else dev, **kw)
    torch.cuda.synchronize()
    xs = x.double().numpy()
    ref, size = xs @ w.T, np.abs(xs) @ np.abs(w).T
    off = np.abs(y.cpu().numpy().reshape(ref.shape).astype(np.float64) - ref)
    bound = (m.cols / 16 + 2 * -(-m.cols // m.group) + 64) * U * size
    assert np.all(off <= bound + 1e-38), (off / (bound + 1e-38)).max()
    return y


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128, 256, 32768])
def test_sizes(group, zeros, dtype):
    print("q4", group, zeros, dtype, flush=True)
    for rows, cols in ((1, 1), (1, 127), (15, 128), (16, 129), (17, 31), (33, 257), (64, 512), (65, 1000), (100, 33), (3, 4099), (130, 2048)):
        m, w, g = make(rows, cols, group, zeros, seed=rows + cols)
        for nb in (1, 2, 5, 16):
            x = torch.from_numpy(g.standard_normal((nb, cols), dtype=np.float32)).to(TYPES[dtype])
            check(m, w, x)


@pytest.mark.parametrize("nb", list(range(1, 17)))
def test_every_batch(nb):
    for rows, cols, group, zeros in ((515, 1111, 64, True), (2050, 300, 128, False), (4, 12000, 128, True)):
        m, w, g = make(rows, cols, group, zeros, seed=nb)
        x = torch.from_numpy(g.standard_normal((nb, cols), dtype=np.float32)).half()
        check(m, w, x)


@pytest.mark.parametrize("shape", [(1024, 8192), (8192, 1024), (20000, 512), (40, 28672), (4100, 3001), (1500, 20000), (2047, 9001), (17, 70001), (13000, 1600)], ids=str)
def test_larger(shape):
    print("q4", shape, flush=True)
    rows, cols = shape
    g = np.random.default_rng(rows)
    groups = -(-cols // 128)
    codes = g.integers(0, 256, (rows, (cols + 1) // 2), dtype=np.uint8)
    scales = (0.001 + 0.01 * g.random((rows, groups))).astype(np.float16)
    m = endor.q4_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), None, cols, 128)
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(rows, -1)[:, :cols]
    w = (c.astype(np.float64) - 8) * np.repeat(scales.astype(np.float64), 128, axis=1)[:, :cols]
    for nb, dtype in ((1, "f16"), (7, "bf16"), (16, "f16")):
        check(m, w, torch.from_numpy(g.standard_normal((nb, cols), dtype=np.float32)).to(TYPES[dtype]))


@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [4100, 8200, 11111, 16001, 20011, 24001, 28001, 32005, 57400])
def test_row_tiles(rows, group, zeros):
    """One row tile to seven of them for a workgroup."""
    print("q4 rows", rows, group, zeros, flush=True)
    m, w, g = make(rows, 900, group, zeros, seed=rows)
    for nb, dtype in ((2, "f16"), (13, "bf16"), (16, "f16")):
        check(m, w, torch.from_numpy(g.standard_normal((nb, 900), dtype=np.float32)).to(TYPES[dtype]))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_strides_and_alignment(dtype):
    """Rows of x at every 2-byte alignment, with NaN between and behind them, and y between guards."""
    for rows, cols, group, zeros in ((50, 200, 32, True), (33, 131, 128, False)):
        m, w, g = make(rows, cols, group, zeros, seed=9)
        for nb in (1, 3, 16):
            x = torch.from_numpy(g.standard_normal((nb, cols), dtype=np.float32)).to(TYPES[dtype])
            for off, pitch in ((0, cols + 8 - cols % 8), (1, cols + 1), (3, cols), (4, cols + 13)):
                buf = torch.full((off + nb * pitch + 64,), float("nan"), dtype=TYPES[dtype], device="cuda")
                dev = torch.as_strided(buf, (nb, cols), (pitch, 1), off)
                dev.copy_(x)
                guard = torch.full((nb * rows + 32,), -7.0, device="cuda")
                y = guard[16:16 + nb * rows].view(nb, rows)
                check(m, w, x, dev=dev, Y=y)
                assert torch.all(guard[:16] == -7) and torch.all(guard[16 + nb * rows:] == -7)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_exact_on_whole_numbers(dtype):
    """Scales of one and whole inputs: every sum is a whole number below 2^24, so the result is exact."""
    g = np.random.default_rng(3)
    rows, cols, group = 70, 900, 64
    codes = g.integers(0, 256, (rows, cols // 2), dtype=np.uint8)
    z = g.integers(0, 16, (rows, 15), dtype=np.uint8)
    scales = np.ones((rows, 15), np.float16)
    m = endor.q4_pack(*(torch.from_numpy(a).cuda() for a in (codes, scales, z)), cols, group)
    w = orc.q4_dense(codes, scales, z, cols, group)
    for nb in (1, 4, 16):
        x = torch.from_numpy(g.integers(-100, 101, (nb, cols)).astype(np.float32)).to(TYPES[dtype])
        y = endor.q4_gemm(m, x.cuda())
        assert np.array_equal(y.cpu().numpy().astype(np.float64), x.double().numpy() @ w.T)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_large_and_small_inputs_keep_their_weights(dtype):
    """A huge x under a weight of zero takes nothing from the small ones; subnormal inputs count in full."""
    rows, cols, group = 20, 256, 64
    codes = np.full((rows, cols // 2), 0x88, np.uint8)
    g = np.random.default_rng(4)
    codes[:, 1::2] = g.integers(0, 256, (rows, cols // 4), dtype=np.uint8)
    scales = np.full((rows, 4), 0.5, np.float16)
    m = endor.q4_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), None, cols, group)
    w = orc.q4_dense(codes, scales, None, cols, group)
    big, small = (60000.0, 2.0 ** -24) if dtype == "f16" else (1e38, 1e-30)
    x = np.zeros((2, cols), np.float32)
    at = np.arange(cols) // 2 % 2 == 0
    x[:, at] = big
    x[0, ~at] = small * g.integers(1, 9, (~at).sum())
    x[1, ~at] = g.standard_normal((~at).sum())
    check(m, w, torch.from_numpy(x).to(TYPES[dtype]))


def test_not_finite_inputs():
    m, w, g = make(40, 300, 64, True, seed=5)
    x = torch.from_numpy(g.standard_normal((3, 300), dtype=np.float32)).half()
    x[1, 299] = float("nan")
    x[2, 0] = float("inf")
    y = endor.q4_gemm(m, x.cuda()).cpu().numpy()
    ref = x.double().numpy() @ w.T
    assert np.all(np.isfinite(y[0])) and np.all(np.isnan(y[1]))
    with np.errstate(invalid="ignore"):
        ref[2] = (x[2].double().numpy()[None] * w).sum(1)
    assert np.array_equal(np.isnan(y[2]), np.isnan(ref[2])) and np.array_equal(np.isinf(y[2]), np.isinf(ref[2]))


def test_empty():
    m, w, g = make(5, 64, 32, True)
    assert endor.q4_gemm(m, torch.zeros((0, 64), dtype=torch.float16, device="cuda")).shape == (0, 5)
    none = endor.Q4Matrix(7, 0, 32, False, torch.empty(0, dtype=torch.uint8, device="cuda"))
    y = endor.q4_gemm(none, torch.zeros((3, 0), dtype=torch.float16, device="cuda"), Y=torch.full((3, 7), 5.0, device="cuda"))
    assert torch.all(y == 0)


@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
def test_quantize(zeros):
    """Every code is the nearest one to its value under the group's rounded scale, and none is off by more than the scale says."""
    g = np.random.default_rng(7)
    for rows, cols, group in ((5, 64, 32), (3, 1001, 128), (40, 300, 256), (2, 7, 32)):
        dense = (g.standard_normal((rows, cols)) * 0.02).astype(np.float16)
        dense[0, :min(cols, group)] = 0
        if cols > 40:
            dense[1, :] = np.abs(dense[1, :])
            dense[-1, :] = -np.abs(dense[-1, :]) if rows > 2 else dense[-1, :]
        codes, scales, points = endor.q4_quantize(torch.from_numpy(dense).cuda(), group, zeros)
        assert (points is not None) == zeros
        c, s = codes.cpu().numpy(), scales.cpu().numpy()
        z = None if points is None else points.cpu().numpy()
        w = orc.q4_dense(c, s, z, cols, group)
        wide = np.repeat(s.astype(np.float64), group, axis=1)[:, :cols]
        # half a step, and where a zero point was rounded or a scale came out below the range's share, what that moves the ends by
        assert np.all(np.abs(w - dense) <= wide * (1.01 if zeros else 0.51) + 1e-7)
        assert z is None or z.max() <= 15
        for i in range(rows):
            for gi in range(s.shape[1]):
                x = dense[i, gi * group:(gi + 1) * group].astype(np.float64)
                want = (max(x.max(), 0) - min(x.min(), 0)) / 15 if zeros else np.abs(x).max() / 7
                assert abs(float(s[i, gi]) - want) <= want * 2.0 ** -10 + 2.0 ** -24


@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128, 256, 512, 1024, 32768])
def test_quantize_every_group(group, zeros):
    """Codes, scales and zero points exactly: the definition takes one fp32 step after the other."""
    g = np.random.default_rng(group)
    for rows, cols in ((1, 1), (3, 33), (67, 1031), (5, 2048), (2, 70001)):
        print("quantize", rows, cols, flush=True)
        dense = (g.standard_normal((rows, cols)) * 0.02).astype(np.float16)
        dense[0, :min(cols, group)] = 0
        codes, scales, points = endor.q4_quantize(torch.from_numpy(dense).cuda(), group, zeros)
        groups = -(-cols // group)
        x = np.zeros((rows, groups * group), np.float32)
        x[:, :cols] = dense
        x = x.reshape(rows, groups, group)
        lo, hi = np.minimum(x.min(2), 0), np.maximum(x.max(2), 0)
        s = ((hi - lo) / np.float32(15) if zeros else np.maximum(hi, -lo) / np.float32(7)).astype(np.float16)
        with np.errstate(divide="ignore"):
            inverse = np.where(s > 0, np.float32(1) / s.astype(np.float32), np.float32(0)).astype(np.float32)
        z = np.clip(np.rint(-lo * inverse), 0, 15) if zeros else np.full_like(inverse, 8)
        c = np.clip(np.rint(x * inverse[..., None]) + z[..., None], 0, 15).astype(np.uint8).reshape(rows, -1)
        c[:, cols:] = 0
        both = c[:, :(cols + 1) // 2 * 2]
        assert np.array_equal(scales.cpu().numpy(), s)  # of the two zeros either
        assert points is None or np.array_equal(points.cpu().numpy(), z.astype(np.uint8))
        assert np.array_equal(codes.cpu().numpy(), both[:, 0::2] | both[:, 1::2] << 4)


def test_refusals():
    m, w, g = make(16, 128, 64, True)
    x = torch.zeros((2, 128), dtype=torch.float16, device="cuda")
    for bad in (x.float(), x[:, :64], x.cpu(), x[0]):
        with pytest.raises(ValueError):
            endor.q4_gemm(m, bad)
    with pytest.raises(ValueError):
        endor.q4_gemm(m, x, Y=torch.empty((2, 16), dtype=torch.float16, device="cuda"))
    with pytest.raises(endor.EndorError):
        endor.q4_gemm(m, torch.zeros((17, 128), dtype=torch.float16, device="cuda"))
    codes, scales = torch.zeros((4, 64), dtype=torch.uint8, device="cuda"), torch.zeros((4, 2), dtype=torch.float16, device="cuda")
    for bad in ((codes[:, :60], scales, None, 128, 64), (codes, scales.float(), None, 128, 64), (codes, scales[:, :1], None, 128, 64),
                (codes, scales, scales, 128, 64), (codes.cpu(), scales.cpu(), None, 128, 64), (codes, scales, None, 128, 0)):
        with pytest.raises(ValueError):
            endor.q4_pack(*bad)
    with pytest.raises(endor.EndorError):
        endor.q4_pack(codes, torch.zeros((4, 3), dtype=torch.float16, device="cuda"), None, 128, 48)
