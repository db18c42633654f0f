"""The mean of the aggregation step on microscaled 4-bit codes: the integer sum
times 2^(e - 1) over M, rounded once, for every number of workers.

The expected value divides in 64 bits and rounds to 32.  That is one rounding:
x = s / M with |s| < 2^31 and 12 M < 2^31 is a binary32 midpoint (25 bits, j /
2^t) or differs from it by at least 1 / (M 2^t) = x / (M j) > 2^-52.5 x, more
than the 2^-53 x by which 64 bits are off; scaling by a power of two is exact
in 64 bits, and below 2^-126 the midpoints have fewer bits still."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2109_12497_amd as uq  # noqa: E402
from paper_2109_12497_amd.mx4 import Mx4Step  # noqa: E402

DEV = torch.device("cuda:0")


def rounded_once(total, scale_bytes, M):
    b = np.repeat(scale_bytes.astype(np.int64), 32)[:total.size]
    with np.errstate(over="ignore"):
        return (total.astype(np.float64) / M * 2.0 ** (b - 128.0)).astype(np.float32)


def gradients(M, d, seed):
    """Blocks of every width, denormal ones and those next to the largest number included."""
    rng = np.random.default_rng(seed)
    g = rng.normal(size=(M, d)) * 2.0 ** np.repeat(rng.integers(-149, 124, size=-(-d // 32)), 32)[:d]
    return np.clip(g, -3e38, 3e38).astype(np.float32)


@pytest.mark.parametrize("M", [1, 2, 3, 5, 6, 7, 9, 10, 11, 13, 14, 15, 16, 17, 33, 100])
@pytest.mark.parametrize("d", [1000, 300_000])
def test_every_form_rounds_once(M, d):
    if M > 16 and d > 1000:
        d = 20_000
    host = gradients(M, d, M)
    g = torch.zeros((M, -(-d // 64) * 64), device=DEV)
    g[:, :d] = torch.from_numpy(host).to(DEV)
    for streamed in (False, True):
        st = Mx4Step(d, M, device=DEV, streamed=streamed)
        out = st.run(g, M)
        torch.cuda.synchronize()
        want = rounded_once(st.sum[:d].cpu().numpy(), st.scales[:-(-d // 32)].cpu().numpy(), M)
        assert np.array_equal(out.cpu().numpy().view(np.int32), want.view(np.int32))


@pytest.mark.parametrize("d,M", [(12_100_003, 3), (12_600_001, 7), (11_000_000, 12)])
def test_large_steps_round_once(d, M):
    """The forms whose outputs pass the caches by."""
    g = torch.empty((M, -(-d // 64) * 64), device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(M)
    for m in range(M):
        g[m].normal_(generator=gen)
    st = Mx4Step(d, M, device=DEV)
    out = st.run(g, 1)
    torch.cuda.synchronize()
    want = rounded_once(st.sum[:d].cpu().numpy(), st.scales[:-(-d // 32)].cpu().numpy(), M)
    assert np.array_equal(out.cpu().numpy().view(np.int32), want.view(np.int32))


@pytest.mark.parametrize("M", [3, 7, 1000, 65_537, 3_000_001, 178_956_970])
def test_sums_that_a_program_holds(M):
    """Sums up to 12 M that came from elsewhere, one row of zeros added to them:
    beyond 2^24 they are no binary32 numbers, and some quotients are ties."""
    d = 32 * 128
    rng = np.random.default_rng(M)
    total = rng.integers(-12 * M, 12 * M + 1, size=d).astype(np.int32)
    total[:64] = np.arange(-32, 32)
    total[64:128] = np.clip(np.arange(64, dtype=np.int64) * M // 5, -12 * M, 12 * M)
    k = 2 * rng.integers(1 << 23, 1 << 24, size=128).astype(np.int64) + 1  # 25 bits: ties where they fit
    total[128:256] = np.where(k * 3 <= 12 * M, k * 3, 5)
    b = rng.integers(1, 253, size=d // 32).astype(np.uint8)
    b[:16] = 1
    s = torch.from_numpy(total).to(DEV)
    out = torch.zeros(d, device=DEV)
    uq.uq_mx4_quantize_sum(torch.zeros((1, d), device=DEV), d, 1, d, 0, torch.from_numpy(b).to(DEV), 1, 1, s, M, out)
    torch.cuda.synchronize()
    assert np.array_equal(s.cpu().numpy(), total)
    assert np.array_equal(out.cpu().numpy().view(np.int32), rounded_once(total, b, M).view(np.int32))
