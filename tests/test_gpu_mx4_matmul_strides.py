"""The product of microscaled 4-bit matrices whose rows lie far apart: up to 2^23
bytes a tile's rows are within a buffer's 2^31 bytes, beyond, the form that
addresses every row by 64 bits is taken whatever the sizes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2109_12497_amd as uq  # noqa: E402
from launches import captured  # noqa: E402
from test_gpu_mx4_matmul import DEV, new_out, operand  # noqa: E402

MOST = 1 << 23


# tiles of 64 x 128, 128 x 128 in parts, 256 x 256
@pytest.mark.parametrize("m,n,k", [(192, 4096, 4096), (700, 900, 9001), (5003, 4099, 300)])
@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_which_form_is_launched(m, n, k, which):
    """Captured, never run: a stride is a number until then."""
    some = torch.zeros(1 << 12, dtype=torch.uint8, device=DEV)
    ws = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    for ld, form in ((MOST, "k_mx4_tiles"), (MOST + 16, "k_mx4_rows_by")):
        lds = [ld if i == which else 8192 for i in range(4)]  # of a, its scales, b, its scales
        kernels = captured(lambda: uq.uq_mx4_matmul(some, lds[0], some, lds[1], some, lds[2], some, lds[3], m, n, k,
                                                    uq.UQ_F32, some, 8192, 0, ws, ws.numel()))
        assert any(form in name for name, _ in kernels), kernels
        assert all("k_mx4_tiles" not in name for name, _ in kernels) or form == "k_mx4_tiles", kernels


def far_apart(t, ld):
    """The rows of t, ld bytes apart, with 0xFF between them."""
    wide = torch.full((t.shape[0], ld), 0xFF, dtype=torch.uint8, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide


@pytest.mark.parametrize("ld", [MOST, MOST + 16])
@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_products_of_rows_far_apart(ld, which):
    m, n, k = (130, 9000, 513) if which < 2 else (9000, 130, 513)
    rng = np.random.default_rng(which)
    a, b = operand(m, k, rng, 126, 128, 0), operand(n, k, rng, 126, 128, 0)
    parts = [a[0], a[1], b[0], b[1]]
    parts[which] = far_apart(parts[which], ld)
    out = new_out(m, n, "fp32")
    ws = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    uq.uq_mx4_matmul(*(v for t in parts for v in (t, t.stride(0))), m, n, k, uq.UQ_F32, out, out.stride(0), 0, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(out[:, :n].cpu().double(), torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t())
    assert (out[:, n:] == -3.0).all()
