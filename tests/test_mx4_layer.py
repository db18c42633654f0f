"""What the microscaled layer and step refuse, without a GPU."""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2109_12497_amd", reason="libuq.so not built")

from paper_2109_12497_amd.mx4 import Mx4Linear, Mx4Step  # noqa: E402
from paper_2109_12497_amd import sgd  # noqa: E402


@pytest.mark.parametrize("kw", [dict(tokens=0), dict(inputs=0), dict(outputs=0), dict(dtype=torch.float64)])
def test_layer_shapes(kw):
    with pytest.raises(AssertionError):
        Mx4Linear(**{**dict(tokens=4, inputs=8, outputs=16, device="cpu"), **kw})


def test_layer_arguments():
    layer = Mx4Linear(4, 40, 16, device="cpu")
    x = torch.zeros(4, 40)
    for bad in (torch.zeros(5, 40), torch.zeros(4, 39), x.double(), torch.zeros(40, 4).t(), torch.zeros(4, 40, 1)):
        with pytest.raises(AssertionError):
            layer.forward(bad)
    for bad in (torch.zeros(40, 16), torch.zeros(16, 40).to(torch.int32)):
        with pytest.raises(AssertionError):
            layer.load(bad)
    with pytest.raises(AssertionError):
        layer.backward(torch.zeros(4, 16), 1)  # no forward before it
    layer.rows = 4
    for bad in (torch.zeros(3, 16), torch.zeros(4, 15)):
        with pytest.raises(AssertionError):
            layer.backward(bad, 1)
    with pytest.raises(AssertionError):
        Mx4Linear(4, 40, 16, device="cpu", train=False).backward(torch.zeros(4, 16), 1)


def test_step_arguments():
    with pytest.raises(AssertionError):
        Mx4Step(10, 0, device="cpu")
    step = Mx4Step(100, 2, device="cpu")
    for bad in (torch.zeros(3, 128), torch.zeros(2, 64), torch.zeros(2, 128).double(), torch.zeros(128, 2).t()):
        with pytest.raises(AssertionError):
            step.run(bad, 1)


def test_variance_bound():
    """The microscaled bound is the smaller of its two terms and falls with the workers."""
    p4, p16 = (sgd.make_problem(n=32, M=M, rows=64, seed=1) for M in (4, 16))
    b4, b16 = sgd.variance_bound(p4, sgd.MX4) / p4.W_max ** 2, sgd.variance_bound(p16, sgd.MX4) / p16.W_max ** 2
    assert b16 < b4 <= 32 / 9
    assert b4 == pytest.approx((1 / 16 + (32 * 4) ** 0.5 / 6) / 4)
