"""Quantisation to microscaled 4-bit floating point and reading it back, bit
for bit against the 64-bit implementation."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2109_12497_amd as uq  # noqa: E402
from oracle import mx4  # noqa: E402

DEV = torch.device("cuda:0")
DTYPES = {"fp32": (torch.float32, uq.UQ_F32, 4), "bf16": (torch.bfloat16, uq.UQ_BF16, 8),
          "fp16": (torch.float16, uq.UQ_F16, 8)}
FILL = 0xA5


def up(n, m):
    return -(-n // m) * m


def matrix(rows, cols, dtype, seed, pad=0):
    """A device matrix whose rows are apart, NaN past cols (never to be read
    into a result), and its values in 64 bits."""
    tdt, _, mult = DTYPES[dtype]
    rng = np.random.default_rng(seed)
    v = rng.normal(size=(rows, cols)) * 2.0 ** rng.uniform(-6, 3, size=(rows, 1))
    x = torch.full((rows, up(max(cols, 1), mult) + mult * pad), float("nan"), dtype=tdt)
    x[:, :cols] = torch.from_numpy(v).to(tdt)
    return x.to(DEV), x[:, :cols].double().numpy()


def buffers(rows, cols, pad=0):
    codes = torch.full((rows, 16 * -(-cols // 32) + 16 * pad), FILL, dtype=torch.uint8, device=DEV)
    scales = torch.full((rows, up(-(-cols // 32), 16) + 16 * pad), FILL, dtype=torch.uint8, device=DEV)
    return codes, scales


def quantize(x, dtype, cols, stochastic, seed, form="both", pad=0):
    rows, type_id = x.shape[0], DTYPES[dtype][1]
    c, s = buffers(rows, cols, pad) if form != "cols" else (None, None)
    ct, st = buffers(cols, rows, pad) if form != "rows" else (None, None)
    ld = lambda t: 0 if t is None else t.stride(0)  # noqa: E731
    uq.uq_mx4_quantize(x, type_id, rows, cols, x.stride(0), stochastic, seed, c, ld(c), s, ld(s), ct, ld(ct), st, ld(st))
    torch.cuda.synchronize()
    return [None if t is None else t.cpu().numpy() for t in (c, s, ct, st)]


def check(host, got_codes, got_scales, r):
    codes, scales = mx4.quantize(host, r)
    n, nb = codes.shape[1], scales.shape[1]
    assert np.array_equal(got_scales[:, :nb], scales)
    bad = np.argwhere(got_codes[:, :n] != codes)
    assert bad.size == 0, (bad[:3], got_codes[tuple(bad[0])], codes[tuple(bad[0])])
    assert (got_codes[:, n:] == FILL).all() and (got_scales[:, nb:] == FILL).all()  # left as they were


SIZES = [(1, 1), (1, 4096), (2, 7), (3, 8), (5, 31), (31, 32), (32, 33), (33, 64), (64, 65), (127, 96), (128, 128),
         (129, 100), (300, 191), (1000, 40), (4099, 3), (37, 5003)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("stochastic", [0, 1])
def test_both_orientations(rows, cols, dtype, stochastic):
    x, host = matrix(rows, cols, dtype, rows * 7 + cols, pad=rows % 3)
    seed = 0x1234567890 + rows
    c, s, ct, st = quantize(x, dtype, cols, stochastic, seed, pad=cols % 2)
    r = mx4.words(rows, cols, 0, seed) if stochastic else None
    check(host, c, s, r)
    check(host.T, ct, st, None if r is None else r.T)


@pytest.mark.parametrize("form", ["rows", "cols"])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("stochastic", [0, 1])
def test_one_orientation(form, dtype, stochastic):
    rows, cols = 205, 333
    x, host = matrix(rows, cols, dtype, 5)
    c, s, ct, st = quantize(x, dtype, cols, stochastic, 99, form)
    r = mx4.words(rows, cols, 0, 99) if stochastic else None
    if form == "rows":
        check(host, c, s, r)
    else:
        check(host.T, ct, st, None if r is None else r.T)


def special(dtype):
    """Rows of 96 with everything a block can hold."""
    tdt = DTYPES[dtype][0]
    info = torch.finfo(tdt)
    rng = np.random.default_rng(3)
    rows = [np.zeros(96), -np.zeros(96), np.full(96, float(info.tiny)), np.full(96, -float(info.max)),
            rng.normal(size=96) * float(info.tiny), np.where(np.arange(96) % 5 == 0, float(info.max) * 0.7, 1e-3),
            np.tile(np.arange(32) / 8.0, 3), np.tile(-np.arange(32) / 4.0, 3) * 3.0]
    for bad in (np.inf, -np.inf, np.nan):
        for at in (0, 40, 95):
            row = rng.normal(size=96)
            row[at] = bad
            rows.append(row)
    smallest = float(info.smallest_normal) * float(info.eps)  # a denormal
    rows += [np.full(96, smallest), np.where(np.arange(96) == 50, smallest, 0.0), np.r_[np.full(95, smallest), 1.0]]
    while len(rows) % 32:
        rows.append(rng.normal(size=96))
    return torch.from_numpy(np.stack(rows)).to(tdt)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("stochastic", [0, 1])
def test_special_values(dtype, stochastic):
    x = special(dtype)
    host = x.double().numpy()
    c, s, ct, st = quantize(x.to(DEV), dtype, 96, stochastic, 31)
    r = mx4.words(x.shape[0], 96, 0, 31) if stochastic else None
    check(host, c, s, r)
    check(host.T, ct, st, None if r is None else r.T)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_nearest_at_every_boundary(dtype):
    """Each multiple of 1/32 of the scale and its neighbours in the type."""
    tdt = DTYPES[dtype][0]
    base = torch.arange(0, 193, dtype=torch.float64).div(32).to(tdt)
    inf = torch.tensor(float("inf")).to(tdt)
    v = torch.cat([base, torch.nextafter(base, inf), torch.nextafter(base, -inf).abs()])
    v = v[v.double() <= 6.0]
    v = torch.cat([v, -v])
    x = torch.zeros(v.numel(), 32, dtype=tdt)
    x[:, 5], x[:, 9] = v, 6.0
    c, s, _, _ = quantize(x.to(DEV), dtype, 32, 0, 0, "rows")
    check(x.double().numpy(), c, s, None)


def test_stochastic_ties_of_the_high_half():
    """Elements whose thresholds share the high half of their uniform words, so
    that the low halves decide: made from the words themselves."""
    rows, cols, seed = 64, 256, 77
    r = mx4.words(rows, cols, 0, seed)
    for base, step, delta in ((0.0, 0.5, 0), (1.0, 0.5, 1), (2.0, 1.0, -1), (4.0, 2.0, 0)):
        # part = (high half + small) / 2^16 in the grid step above base
        part = ((r >> np.uint64(16)).astype(np.float64) + (delta + 1) * 0.25) / 65536.0
        y = np.minimum(base + step * part, 6.0)
        x = y.astype(np.float32)
        x[:, ::32] = 6.0
        c, s, ct, st = quantize(torch.from_numpy(x).to(DEV), "fp32", cols, 1, seed)
        check(x.astype(np.float64), c, s, r)
        check(x.astype(np.float64).T, ct, st, r.T)


def test_capped_grids_and_streams():
    """On a grid capped at 8 blocks (rows and tiles in many launches), on a
    stream of its own."""
    rows, cols = 700, 1000
    x, host = matrix(rows, cols, "bf16", 8)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    uq.uq_set_grid_cap(8)
    try:
        with torch.cuda.stream(side):
            c, s, ct, st = quantize(x, "bf16", cols, 1, 5)
    finally:
        uq.uq_set_grid_cap(0)
    r = mx4.words(rows, cols, 0, 5)
    check(host, c, s, r)
    check(host.T, ct, st, r.T)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 8), (33, 32), (7, 100), (129, 257), (64, 4096), (1021, 31)])
def test_dequantize(rows, cols, dtype):
    """Random fields on every scale byte, 255 included: the value in 64 bits
    rounded once."""
    tdt, type_id, mult = DTYPES[dtype]
    rng = np.random.default_rng(rows * 1000 + cols)
    nb = -(-cols // 32)
    codes, scales = buffers(rows, cols, 1)
    codes[:, :16 * nb] = torch.from_numpy(rng.integers(0, 256, size=(rows, 16 * nb), dtype=np.uint8))
    b = rng.integers(0, 256, size=(rows, nb), dtype=np.uint8)
    scales[:, :nb] = torch.from_numpy(b)
    out = torch.full((rows, up(cols, mult) + mult), -7.0, dtype=tdt, device=DEV)
    uq.uq_mx4_dequantize(codes, codes.stride(0), scales, scales.stride(0), rows, cols, type_id, out, out.stride(0))
    torch.cuda.synchronize()
    v = mx4.decode(codes[:, :16 * nb].cpu().numpy(), b, cols)
    assert torch.equal(torch.nan_to_num(out[:, :cols].cpu(), nan=12345.0),
                       torch.nan_to_num(torch.from_numpy(v).to(tdt), nan=12345.0))
    assert (out[:, cols:] == -7.0).all()


def test_round_trip_of_what_is_on_the_grid():
    """Values that codes stand for come back bit for bit, rows and transposed."""
    rows, cols = 96, 160
    rng = np.random.default_rng(0)
    f = rng.integers(0, 16, size=(rows, cols)).astype(np.uint8)
    f[::32, :] = 7  # one 6 in each block of either orientation
    f[:, ::32] = 7
    v = torch.from_numpy(mx4.decode(mx4.pack(f), np.full((rows, 5), 125, dtype=np.uint8), cols)).float()
    c, s, ct, st = quantize(v.to(DEV), "fp32", cols, 0, 0)
    assert (s[:, :5] == 125).all() and (st[:, :3] == 125).all()
    assert np.array_equal(c, mx4.pack(f)) and np.array_equal(ct, mx4.pack(np.ascontiguousarray(f.T)))


def test_rows_beyond_2_to_31_bytes():
    """The last row's codes lie past 2^31 and its elements past 2^32 bytes."""
    rows, cols = 3, 8
    ld = (1 << 30) + 512
    x = torch.zeros(2 * ld + 8, dtype=torch.bfloat16, device=DEV)
    v = torch.tensor([1.0, -2.0, 3.0, 6.0, 0.3, -0.6, 1.26, 5.2], dtype=torch.bfloat16)
    for i in range(rows):
        x[i * ld:i * ld + 8] = v.to(DEV) * (i + 1)
    codes = torch.zeros(2 * ld + 16, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(2 * ld + 16, dtype=torch.uint8, device=DEV)
    uq.uq_mx4_quantize(x, uq.UQ_BF16, rows, cols, ld, 0, 0, codes, ld, scales, ld, None, 0, None, 0)
    torch.cuda.synchronize()
    for i in range(rows):
        c, s = mx4.quantize((v * (i + 1)).double().numpy()[None, :], None)
        assert np.array_equal(codes[i * ld:i * ld + 16].cpu().numpy(), c[0])
        assert scales[i * ld].item() == s[0, 0]
    out = torch.zeros(2 * ld + 8, dtype=torch.bfloat16, device=DEV)
    uq.uq_mx4_dequantize(codes, ld, scales, ld, rows, cols, uq.UQ_BF16, out, ld)
    torch.cuda.synchronize()
    assert torch.equal(out[2 * ld:].cpu().double(), torch.from_numpy(mx4.decode(c, s, 8))[0])
