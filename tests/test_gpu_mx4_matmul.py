"""The product of microscaled 4-bit matrices against 64 bits.

Where the operands' scales span few powers of two every partial sum is a
binary32 number, and the result has to be equal bit for bit in any order of
summation.  With scales over a wide range the bound is that of k additions,
each off by at most 2^-23 of its result (a rounding or a truncation):
k * 2^-23 * sum |a b|, and half a step of the output's type."""
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


def up(n, m):
    return -(-n // m) * m


def operand(rows, k, rng, lo, hi, pad):
    """Random fields with scale bytes in [lo, hi]; what lies past the last
    block is filled with 0xFF (a NaN byte there must not enter a result)."""
    nb = -(-k // 32)
    codes = np.full((rows, 16 * nb + 16 * pad), 0xFF, dtype=np.uint8)
    f = rng.integers(0, 16, size=(rows, k)).astype(np.uint8)
    codes[:, :16 * nb] = mx4.pack(f)
    scales = np.full((rows, up(nb, 16) + 16 * pad), 0xFF, dtype=np.uint8)
    scales[:, :nb] = rng.integers(lo, hi + 1, size=(rows, nb))
    v = mx4.decode(codes[:, :16 * nb], scales[:, :nb], k)
    return torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), v


def matmul(a, b, m, n, k, dtype, out, accumulate, ws=None):
    ws = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV) if ws is None else ws
    uq.uq_mx4_matmul(a[0], a[0].stride(0), a[1], a[1].stride(0), b[0], b[0].stride(0), b[1], b[1].stride(0), m, n, k,
                     DTYPES[dtype][1], out, out.stride(0), accumulate, ws, ws.numel())


def new_out(m, n, dtype, pad=0, fill=-3.0):
    tdt, _, mult = DTYPES[dtype]
    return torch.full((m, up(n, mult) + mult * pad), fill, dtype=tdt, device=DEV)


def case(m, n, k, dtype, accumulate, seed, lo=126, hi=128, pad=1):
    rng = np.random.default_rng(seed)
    a, b = operand(m, k, rng, lo, hi, pad), operand(n, k, rng, lo, hi, 0)
    out = new_out(m, n, dtype, pad)
    matmul(a, b, m, n, k, dtype, out, accumulate)
    torch.cuda.synchronize()
    want = torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t() + (-3.0 if accumulate else 0.0)
    return out, want, a, b


SHAPES = [(1, 1, 1), (1, 8, 32), (1, 64, 33), (1, 1000, 4096), (2, 17, 100), (3, 300, 31), (8, 129, 4000), (16, 64, 64),
          (17, 33, 2047), (31, 32, 512), (33, 1025, 96), (64, 64, 128), (65, 127, 1024), (100, 500, 255), (128, 128, 256),
          (129, 260, 257), (255, 256, 4096), (256, 256, 32), (257, 513, 320), (300, 1, 700), (512, 768, 1000), (1100, 40, 64), (3300, 2900, 520)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("accumulate", [0, 1])
def test_exact_sums(m, n, k, accumulate):
    """Multiples of 1/16 up to 4096 * 36 * 4: every partial sum is below 2^24 / 16."""
    out, want, _, _ = case(m, n, k, "fp32", accumulate, m + n * 3 + k)
    assert torch.equal(out[:, :n].cpu().double(), want)
    assert (out[:, n:] == -3.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", [(1, 1000, 512), (7, 65, 97), (33, 40, 1000), (130, 257, 256), (512, 512, 512)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_narrow_outputs(m, n, k, dtype, accumulate):
    """The exact sum rounded once (k * 36 * 4 at most 147456: beyond fp16's
    65504 only as an infinity, which the rounding gives too)."""
    out, want, _, _ = case(m, n, k, dtype, accumulate, m * 5 + n + k)
    assert torch.equal(out[:, :n].cpu(), want.to(DTYPES[dtype][0]))
    assert (out[:, n:] == -3.0).all()


@pytest.mark.parametrize("m,n,k", [(1, 200, 5003), (19, 333, 700), (200, 300, 1500), (257, 129, 9000)])
def test_wide_scales(m, n, k):
    out, want, a, b = case(m, n, k, "fp32", 0, k, lo=100, hi=150)
    size = torch.from_numpy(np.abs(a[2])) @ torch.from_numpy(np.abs(b[2])).t()
    assert (torch.abs(out[:, :n].cpu().double() - want) <= k * 2.0 ** -23 * size + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("m,n,k", [(1, 70, 100), (5, 40, 257), (140, 270, 500)])
def test_extreme_scales(m, n, k):
    """Bytes 1 and 253 against their opposites: 2^-126 * 2^126 = 1."""
    rng = np.random.default_rng(m)
    a, b = list(operand(m, k, rng, 1, 1, 0)), list(operand(n, k, rng, 253, 253, 0))
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :n].cpu().double(), torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t())


@pytest.mark.parametrize("m,n,k", [(1, 50, 200), (40, 50, 200), (270, 300, 600)])
def test_nan_blocks_reach_their_rows_and_columns_alone(m, n, k):
    rng = np.random.default_rng(m + 1)
    a, b = operand(m, k, rng, 127, 127, 1), operand(n, k, rng, 127, 127, 0)
    a[1][m // 2, 3] = 255
    b[1][n - 1, 0] = 255
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    want = torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t()
    want[m // 2, :] = float("nan")
    want[:, n - 1] = float("nan")
    assert torch.equal(torch.nan_to_num(out[:, :n].cpu().double(), nan=1e30), torch.nan_to_num(want, nan=1e30))


@pytest.mark.parametrize("m,n,k", [(4, 30, 0), (300, 300, 0)])
def test_no_terms(m, n, k):
    empty = torch.zeros((max(m, n), 16), dtype=torch.uint8, device=DEV)
    for accumulate, value in ((0, 0.0), (1, -3.0)):
        out = new_out(m, n, "bf16")
        matmul((empty, empty), (empty, empty), m, n, k, "bf16", out, accumulate)
        torch.cuda.synchronize()
        assert (out[:, :n] == value).all()


@pytest.mark.parametrize("m,n,k", [(1, 300, 8192), (20, 100, 8192), (300, 200, 4096), (512, 512, 65536)])
def test_same_result_every_time(m, n, k):
    """The order of summation is fixed: repeated calls, and calls with other
    work on the card, give the same bits."""
    rng = np.random.default_rng(0)
    a, b = operand(m, k, rng, 100, 150, 0), operand(n, k, rng, 100, 150, 0)
    outs = []
    for i in range(4):
        out = new_out(m, n, "fp32", fill=float(i))
        ws = torch.full((uq.uq_mx4_matmul_workspace_bytes(m, n, k),), 0x55 + i, dtype=torch.uint8, device=DEV)
        matmul(a, b, m, n, k, "fp32", out, 0, ws)
        torch.cuda.synchronize()
        outs.append(out[:, :n].cpu())
    assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_capped_grid():
    """Tiles in many launches."""
    uq.uq_set_grid_cap(8)
    try:
        out, want, _, _ = case(600, 700, 300, "fp32", 0, 3)
        small, small_want, _, _ = case(3, 900, 2000, "fp32", 1, 4)
    finally:
        uq.uq_set_grid_cap(0)
    assert torch.equal(out[:, :700].cpu().double(), want)
    assert torch.equal(small[:, :900].cpu().double(), small_want)


def test_rows_far_apart():
    """Leading dimensions that put the last rows past 2^31 bytes."""
    rng = np.random.default_rng(9)
    m, n, k = 3, 40, 100
    ld = (1 << 30) + 512
    a, b = operand(m, k, rng, 126, 128, 0), operand(n, k, rng, 126, 128, 0)
    wide = [torch.zeros(2 * ld + t.shape[1], dtype=torch.uint8, device=DEV) for t in a[:2]]
    for w, t in zip(wide, a[:2]):
        for i in range(m):
            w[i * ld:i * ld + t.shape[1]] = t[i]
    out = torch.zeros(2 * ld + 64, dtype=torch.float32, device=DEV)
    ws = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    uq.uq_mx4_matmul(wide[0], ld, wide[1], ld, b[0], b[0].stride(0), b[1], b[1].stride(0), m, n, k, uq.UQ_F32, out, ld,
                     0, ws, ws.numel())
    torch.cuda.synchronize()
    want = torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t()
    for i in range(m):
        assert torch.equal(out[i * ld:i * ld + n].cpu().double(), want[i])
