"""A microscaled layer's captured calls whose products split k, and so use the
layer's workspace, replayed between eager calls that need more of it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2109_12497_amd as uq  # noqa: E402
from oracle import mx4  # noqa: E402
from paper_2109_12497_amd.mx4 import Mx4Linear  # noqa: E402

DEV = torch.device("cuda:0")
INPUTS, OUTPUTS = 16384, 1000


def whole(n, seed):
    """[n, INPUTS] of whole numbers that every sum over them holds exactly."""
    return torch.randint(-6, 7, (n, INPUTS), generator=torch.Generator().manual_seed(seed)).float()


def seen(v):
    codes, scales = mx4.quantize(v.numpy(), None)
    return torch.from_numpy(mx4.decode(codes, scales, INPUTS))


def test_replays_between_calls_that_need_more_workspace():
    need = lambda rows: uq.uq_mx4_matmul_workspace_bytes(rows, OUTPUTS, INPUTS)  # noqa: E731
    captured, others = (64, 96), (200, 512, 1064)
    assert 256 < need(captured[0]) < need(captured[1]) < min(need(r) for r in others)
    layer = Mx4Linear(2048, INPUTS, OUTPUTS, device=DEV, train=False)
    w = whole(OUTPUTS, 1)
    values = seen(w).t().contiguous()
    layer.load(w.to(DEV))
    at, held = layer.ws.data_ptr(), layer.ws.numel()
    graphs = []
    for rows in captured:
        x = whole(rows, rows).to(DEV)
        layer.forward(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layer.forward(x)
        graphs.append((graph, x, y))
    for turn in range(4):
        for i, (graph, x, y) in enumerate(graphs):
            fresh = whole(x.shape[0], 100 + 10 * turn + i)
            x.copy_(fresh)
            y.fill_(-1.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y.cpu().double(), seen(fresh) @ values)
            rows = others[(turn + i) % len(others)]
            other = whole(rows, turn)
            got = layer.forward(other.to(DEV))
            torch.cuda.synchronize()
            assert torch.equal(got.cpu().double(), seen(other) @ values)
    assert layer.ws.data_ptr() == at and layer.ws.numel() == held


def test_captured_backward_whose_weight_gradient_is_split():
    """dw = dy^T x over 12,000 rows is split along them; captured, then run
    eagerly at other numbers of rows in between."""
    tokens, inputs, outputs = 12_000, 96, 80
    assert uq.uq_mx4_matmul_workspace_bytes(outputs, inputs, tokens) > 256
    layer = Mx4Linear(tokens, inputs, outputs, device=DEV)
    gen = torch.Generator().manual_seed(5)
    w, x, dy = (torch.randint(-6, 7, shape, generator=gen).float().to(DEV) for shape in
                ((outputs, inputs), (tokens, inputs), (tokens, outputs)))
    layer.load(w)

    def step(rows, seed):
        layer.forward(x[:rows])
        return layer.backward(dy[:rows], seed=seed)

    ref = [t.clone() for t in step(tokens, 7)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(tokens, 7)
    for rows in (9_000, 1, 11_999, 64):
        for t in outs:
            t.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, r) for t, r in zip(outs, ref))
        _, dw = step(rows, rows)
        torch.cuda.synchronize()
        r = mx4.words(rows, outputs, 0, rows)
        a, b = dy[:rows].cpu().numpy(), x[:rows].cpu().numpy()
        ca, sa = mx4.quantize(np.ascontiguousarray(a.T), r.T)
        cb, sb = mx4.quantize(np.ascontiguousarray(b.T), None)
        va, vb = mx4.decode(ca, sa, rows), mx4.decode(cb, sb, rows)
        # whole numbers and sums of at most 36 * 12000, which binary32 holds
        assert torch.equal(dw.cpu().double(), torch.from_numpy(va @ vb.T))
