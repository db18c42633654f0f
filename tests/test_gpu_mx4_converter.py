"""Rounding to the nearest microscaled code for every 16-bit value, on scales
from the smallest to the largest that a block takes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_mx4 import DEV, DTYPES, check, quantize  # noqa: E402


def every_value(tdt):
    """All 65,536 bit patterns as [2048, 32]: neighbours share a block."""
    return torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16).view(tdt).view(2048, 32)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_value_among_its_neighbours(dtype):
    x = every_value(DTYPES[dtype][0])
    c, s, ct, st = quantize(x.to(DEV), dtype, 32, 0, 0)
    check(x.double().numpy(), c, s, None)
    check(x.double().numpy().T, ct, st, None)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("above", [0, 1, 2, 3])
def test_every_value_below_a_larger_one(dtype, above):
    """Each finite bf16 or fp16 value beside one 1.5 * 2^above times as large as its
    power of two, so that it takes every place of the grid on every scale."""
    tdt = torch.bfloat16 if dtype == "fp32" else DTYPES[dtype][0]
    v = every_value(tdt).flatten()
    v = v[torch.isfinite(v)]
    top = torch.exp2(torch.floor(torch.log2(v.double().abs().clamp(min=2.0 ** -140)))) * 1.5 * 2.0 ** above
    x = torch.zeros(v.numel(), 32, dtype=DTYPES[dtype][0])
    x[:, 7] = v.to(x.dtype)
    x[:, 20] = top.clamp(max=float(torch.finfo(x.dtype).max)).to(x.dtype)
    c, s, _, _ = quantize(x.to(DEV), dtype, 32, 0, 0, "rows")
    check(x.double().numpy(), c, s, None)


@pytest.mark.parametrize("byte", [1, 2, 3, 64, 126, 127, 128, 190, 251, 252, 253])
def test_boundaries_on_a_scale(byte):
    """The middles between codes and their binary32 neighbours, on one scale."""
    e = byte - 127
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 0.0])
    with np.errstate(over="ignore"):
        y = np.ldexp(mid, e).astype(np.float32)
        up, down = np.nextafter(y, np.float32(np.inf)), np.nextafter(y, np.float32(0))
    v = np.concatenate([y, up, down])
    v = v[np.isfinite(v) & (np.abs(v.astype(np.float64)) <= 6.0 * 2.0 ** e)]
    v = np.concatenate([v, -v])
    x = np.zeros((v.size, 32), dtype=np.float32)
    top = np.float32(np.ldexp(6.0, e)) if byte < 253 else np.finfo(np.float32).max
    x[:, 3], x[:, 11] = v, top
    c, s, _, _ = quantize(torch.from_numpy(x).to(DEV), "fp32", 32, 0, 0, "rows")
    assert (s[:, 0] == byte).all()
    check(x.astype(np.float64), c, s, None)
