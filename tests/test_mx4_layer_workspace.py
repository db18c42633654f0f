"""The memory that a microscaled layer holds over calls of every number of
rows, and the workspace it hands to its products, without a GPU."""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2109_12497_amd", reason="libuq.so not built")

import paper_2109_12497_amd as uq  # noqa: E402
from paper_2109_12497_amd import mx4  # noqa: E402


def held_bytes(layer):
    """Bytes of every tensor that the layer keeps, in lists and code buffers too."""
    seen, todo = {}, [vars(layer)]
    while todo:
        v = todo.pop()
        if isinstance(v, torch.Tensor):
            seen[v.untyped_storage().data_ptr()] = v.untyped_storage().nbytes()
        elif isinstance(v, dict):
            todo += v.values()
        elif isinstance(v, (list, tuple, set)):
            todo += v
        elif isinstance(v, mx4.Codes):
            todo.append(vars(v))
    return sum(seen.values())


@pytest.fixture
def calls(monkeypatch):
    """(m, n, k, workspace address, its bytes) of every product, none of which runs."""
    made = []
    monkeypatch.setattr(mx4, "_check_matrix", lambda *a: None)
    monkeypatch.setattr(mx4, "_stream", lambda s: 0)
    monkeypatch.setattr(mx4, "quantize", lambda *a, **k: None)
    monkeypatch.setattr(mx4, "uq_mx4_matmul", lambda *a: made.append((*a[8:11], a[15].data_ptr(), a[16])))
    return made


# with 16384 inputs and 1000 outputs more rows need more workspace up to 1064
# rows, and none from 1536 on; the last is the weight gradient's, over the rows
@pytest.mark.parametrize("tokens,inputs,outputs,train", [(1600, 16384, 1000, False), (200, 4096, 300, True),
                                                         (300, 64, 8192, True), (12_000, 96, 80, True)])
def test_every_number_of_rows_in_one_workspace(calls, tokens, inputs, outputs, train):
    layer = mx4.Mx4Linear(tokens, inputs, outputs, device="cpu", train=train)
    held, at = held_bytes(layer), layer.ws.data_ptr()
    step = 1 if tokens < 2000 else 37
    for rows in range(0, tokens + 1, step):
        layer.forward(torch.empty(rows, inputs))
        if train:
            layer.backward(torch.empty(rows, outputs), seed=rows)
    assert len(calls) == (3 if train else 1) * len(range(0, tokens + 1, step))
    for m, n, k, ws, size in calls:
        assert ws == at and size >= uq.uq_mx4_matmul_workspace_bytes(m, n, k)
    assert held_bytes(layer) == held


def test_no_more_than_the_largest_need():
    layer = mx4.Mx4Linear(1600, 16384, 1000, device="cpu", train=False)
    need = [uq.uq_mx4_matmul_workspace_bytes(rows, 1000, 16384) for rows in range(1, 1601)]
    assert layer.ws.numel() == max(need) > need[-1]
