"""Products of microscaled 4-bit matrices at the ends of binary32: denormal
sums are exact, and what passes the largest number is not finite."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from oracle import mx4  # noqa: E402
from test_gpu_mx4_matmul import DEV, matmul, new_out, operand, up  # noqa: E402

# few rows, few rows of several fragments, tiles of each size, k in parts
SHAPES = [(1, 40, 64), (40, 300, 64), (192, 4096, 256), (700, 900, 9001), (5003, 4099, 40)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("byte", [127, 110, 106])
def test_denormal_sums(m, n, k, byte):
    """Byte 1 against `byte`: products are multiples of 2^-126 * 2^(byte - 127) / 4, at
    least 2^-149, and with 9001 of at most 36 far below 2^24 of those."""
    rng = np.random.default_rng(m + byte)
    a, b = operand(m, k, rng, 1, 1, 0), operand(n, k, rng, byte, byte, 0)
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :n].cpu().double(), torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t())


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_zeros_times_the_largest_scales(m, n, k):
    rng = np.random.default_rng(m)
    a, b = operand(m, k, rng, 253, 253, 0), operand(n, k, rng, 253, 253, 0)
    a[0].fill_(0)
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    assert (out[:, :n] == 0.0).all()


def single(rows, k, at, field, byte):
    """One element a row, the rest zeros."""
    f = np.zeros((rows, k), dtype=np.uint8)
    f[:, at] = field
    scales = np.zeros((rows, up(-(-k // 32), 16)), dtype=np.uint8)
    scales[:, at // 32] = byte
    return torch.from_numpy(mx4.pack(f)).to(DEV), torch.from_numpy(scales).to(DEV), None


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_what_passes_the_largest_number(m, n, k):
    """36 * 2^122 is below it, 36 * 2^123 is not; nor are sums of such of both
    signs, but where they cancel."""
    at = k // 2
    for sa, sb, sign in ((7, 7, 1), (15, 7, -1), (15, 15, 1)):
        for byte, want in ((249, 36.0 * 2.0 ** 122), (250, float("inf"))):
            out = new_out(m, n, "fp32")
            matmul(single(m, k, at, sa, byte), single(n, k, at, sb, 127), m, n, k, "fp32", out, 0)
            torch.cuda.synchronize()
            assert (out[:, :n] == sign * want).all()
    rng = np.random.default_rng(1)
    a, b = operand(m, k, rng, 253, 253, 0), operand(n, k, rng, 140, 140, 0)
    a[0].bitwise_or_(0x77).bitwise_and_(0x7F)  # magnitudes of 6, whole blocks of them
    b[0].bitwise_or_(0x77)
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    # products are +-36 * 2^139 (whole blocks, past k too): a finite sum has as many of either sign
    signs = []
    for codes, rows in ((a[0], m), (b[0], n)):
        f = torch.stack([codes & 15, codes >> 4], dim=-1).view(rows, -1)
        signs.append(torch.where(f > 7, -1.0, 1.0).double().cpu())
    balance = signs[0] @ signs[1].t()
    got = out[:, :n].cpu()
    assert not torch.isfinite(got[balance != 0]).any()
    assert (got[torch.isfinite(got)] == 0.0).all()
