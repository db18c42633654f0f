"""The one-call step on microscaled 4-bit codes at both sides of every change
of its kernel: rows spread over waves or not, outputs and gradients past the
caches or not, 2, 4, 8 or 16 rows in registers."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from oracle import mx4  # noqa: E402
from paper_2109_12497_amd.mx4 import Mx4Step  # noqa: E402

DEV = torch.device("cuda:0")
SPREAD, OUT, GRAD = 1 << 18, 46 << 18, 256 << 18  # coordinates, of one output, of all gradients


@pytest.mark.parametrize("d,M", [(SPREAD, 1), (SPREAD + 1, 1), (SPREAD, 2), (SPREAD + 1, 2), (SPREAD + 1, 3),
                                 (SPREAD + 1, 4), (SPREAD + 1, 5), (OUT, 4), (OUT + 1, 2), (OUT + 1, 4), (OUT, 5),
                                 (OUT + 1, 5), (12_100_003, 5), (GRAD // 5 + 1, 5), (GRAD // 3, 3), (GRAD // 3 + 1, 3),
                                 (GRAD // 2 + 1, 2), (OUT, 16), (OUT + 1, 9), (OUT + 1, 16)])
def test_one_call_and_separate_calls(d, M):
    """Equal everywhere, and at the start and the end to the 64-bit implementation."""
    ldg = -(-d // 64) * 64
    g = torch.empty((M, ldg), device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(M)
    for m in range(M):
        g[m].normal_(generator=gen)
    one, two = Mx4Step(d, M, device=DEV), Mx4Step(d, M, device=DEV, streamed=True)
    one.run(g, 5)
    two.run(g, 5)
    torch.cuda.synchronize()
    assert torch.equal(one.scales, two.scales) and torch.equal(one.sum, two.sum) and torch.equal(one.out, two.out)
    head = 4096
    b, total, out = mx4.aggregate(g[:, :head].cpu().numpy(), head, 5)
    assert np.array_equal(one.scales[:b.size].cpu().numpy(), b)
    assert np.array_equal(one.sum[:head].cpu().numpy(), total)
    assert np.array_equal(one.out[:head].cpu().numpy().view(np.int32), out.view(np.int32))
    assert not one.sum[d:].any() and not one.out[d:].any()
