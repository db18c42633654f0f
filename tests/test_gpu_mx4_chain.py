"""Two microscaled layers one after another: their gradients are without bias
where each backward pass takes a seed of its own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from oracle import mx4  # noqa: E402
from paper_2109_12497_amd.mx4 import Mx4Linear  # noqa: E402

DEV = torch.device("cuda:0")


def test_gradients_through_two_layers():
    """dy through a second layer of weight 1.5 on the diagonal, then through a
    first of weight 1: dx is dy * 1.5 rounded twice.  Its mean over n steps
    against that: an element's deviation is at most half of the widest gap of
    each rounding, 2^e and 2^e', where 6 * 2^e bounds a block of dy and 9 * 2^e
    what the second rounding sees, so that e' <= e + 1; six deviations of the mean."""
    tokens, width, layers, n = 64, 64, 2, 400
    eye = torch.eye(width, device=DEV)
    first, second = (Mx4Linear(tokens, width, width, device=DEV) for _ in range(layers))
    first.load(eye)
    second.load(1.5 * eye)
    x = torch.ones(tokens, width, device=DEV)
    second.forward(first.forward(x))
    dyh = np.random.default_rng(3).normal(size=(tokens, width)).astype(np.float32)
    dy = torch.from_numpy(dyh).to(DEV)
    total = torch.zeros(tokens, width, dtype=torch.float64, device=DEV)
    for step in range(n):
        between, _ = second.backward(dy, seed=step * layers + 1)
        total += first.backward(between, seed=step * layers)[0].double()
    e = np.repeat(mx4.bytes_of(mx4.block_max(dyh)).astype(np.float64) - 127, 32, axis=1)
    deviation = 2.0 ** e * np.hypot(1.5, 2.0) / np.sqrt(n)
    off = np.abs(total.cpu().numpy() / n - 1.5 * dyh.astype(np.float64))
    assert (off <= 6 * deviation).all()
    # and of all elements together, whose roundings are independent
    signed = (total.cpu().numpy() / n - 1.5 * dyh.astype(np.float64)) * np.sign(dyh)
    assert abs(signed.sum()) <= 6 * np.sqrt((deviation ** 2).sum())
