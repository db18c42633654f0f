"""The product of microscaled 4-bit matrices in each of its forms, at odd ends
of each: few rows beside many columns (1 to 4 fragments of either operand),
large matrices with ragged edges (tiles of both sizes), tiles whose k is split
in parts, calls at once on two streams, and replays.

The scales span few powers of two, so that every partial sum is a multiple of
1/16 and, with the signs drawn at random, far below 2^20: a binary32 number, and
the result is equal bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2109_12497_amd as uq  # noqa: E402
from test_gpu_mx4_matmul import DEV, case, matmul, new_out, operand  # noqa: E402


# columns on either side of one, two and three blocks of 16 to a compute unit
@pytest.mark.parametrize("n", [4096, 4097, 8191, 8193, 12288, 12289, 16411])
@pytest.mark.parametrize("m", [1, 16, 17, 32, 33, 47, 49, 64])
def test_few_rows_beside_many_columns(m, n):
    out, want, _, _ = case(m, n, 1111, "fp32", 0, m + n)
    assert torch.equal(out[:, :n].cpu().double(), want)
    assert (out[:, n:] == -3.0).all()


# on either side of a tile's edge along each axis, with k shorter than a stage of
# 256, whole stages, and stages that are no multiple of four
@pytest.mark.parametrize("m,n,k", [(300, 5001, 600), (1025, 513, 33), (65, 9000, 513), (129, 20001, 700),
                                   (5003, 4099, 300), (5001, 2003, 257), (2000, 2100, 5000), (130, 10100, 256),
                                   (1100, 1111, 1025), (511, 8193, 1)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_ragged_tiles(m, n, k, dtype):
    out, want, _, _ = case(m, n, k, dtype, 1, m + n + k)
    assert torch.equal(out[:, :n].cpu(), want.to(out.dtype))
    assert (out[:, n:] == -3.0).all()


# tiles of each size, with 2 and 4 stages in LDS, in one part and in several
@pytest.mark.parametrize("m,n,k", [(562, 3199, 197), (519, 1694, 12261), (81, 2668, 9178), (164, 466, 13001),
                                   (588, 4686, 426), (998, 3709, 1993), (355, 1296, 15040), (128, 2726, 14204),
                                   (839, 5586, 283), (2308, 5034, 1066)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_every_tile(m, n, k, dtype, accumulate):
    out, want, _, _ = case(m, n, k, dtype, accumulate, m + n + k)
    assert torch.equal(out[:, :n].cpu(), want.to(out.dtype))
    assert (out[:, n:] == -3.0).all()


# tiles that fill whole rounds, and the last rows or columns in another form
@pytest.mark.parametrize("m,n,k", [(5911, 1325, 16), (674, 11181, 17), (10760, 1624, 16), (6854, 2483, 33),
                                   (9576, 1726, 100), (6736, 2671, 16), (1777, 10176, 16), (8022, 2068, 161),
                                   (3971, 4352, 262), (4103, 4001, 513)])
@pytest.mark.parametrize("dtype,accumulate", [("fp32", 1), ("bf16", 0), ("fp16", 1)])
def test_whole_rounds_and_a_rest(m, n, k, dtype, accumulate):
    out, want, _, _ = case(m, n, k, dtype, accumulate, m + n + k)
    assert torch.equal(out[:, :n].cpu(), want.to(out.dtype))
    assert (out[:, n:] == -3.0).all()


def test_whole_rounds_and_a_split_rest():
    """The last rows' k in parts, which need the workspace."""
    m, n, k = 8400, 2000, 8192
    assert uq.uq_mx4_matmul_workspace_bytes(m, n, k) > 256
    out, want, _, _ = case(m, n, k, "fp32", 1, 6)
    assert torch.equal(out[:, :n].cpu().double(), want)
    assert (out[:, n:] == -3.0).all()


@pytest.mark.parametrize("m,n,k", [(300, 6000, 600), (1000, 1030, 9001), (998, 3709, 1993), (5001, 2003, 257),
                                   (3971, 4352, 262)])
def test_nan_blocks_in_tiles(m, n, k):
    rng = np.random.default_rng(m)
    a, b = operand(m, k, rng, 127, 127, 1), operand(n, k, rng, 127, 127, 0)
    a[1][m // 2, 3] = 255
    b[1][n - 1, (k - 1) // 32] = 255
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    want = torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t()
    want[m // 2, :] = float("nan")
    want[:, n - 1] = float("nan")
    assert torch.equal(torch.nan_to_num(out[:, :n].cpu().double(), nan=1e30), torch.nan_to_num(want, nan=1e30))


@pytest.mark.parametrize("m,n,k", [(140, 9001, 700), (1030, 1000, 9000), (998, 3709, 1993)])
def test_extreme_scales_in_tiles(m, n, k):
    """Bytes 1 and 253 against their opposites: 2^-126 * 2^126 = 1."""
    rng = np.random.default_rng(n)
    a, b = operand(m, k, rng, 1, 1, 0), operand(n, k, rng, 253, 253, 0)
    out = new_out(m, n, "fp32")
    matmul(a, b, m, n, k, "fp32", out, 0)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :n].cpu().double(), torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t())


def test_tiles_in_many_launches():
    uq.uq_set_grid_cap(8)
    try:
        large, large_want, _, _ = case(5001, 2003, 257, "fp32", 0, 3)
        split, split_want, _, _ = case(700, 900, 9001, "fp32", 1, 4)
        rows, rows_want, _, _ = case(700, 600, 300, "fp32", 1, 5)
    finally:
        uq.uq_set_grid_cap(0)
    for out, want in ((large, large_want), (split, split_want), (rows, rows_want)):
        assert torch.equal(out[:, :want.shape[1]].cpu().double(), want)


@pytest.mark.parametrize("m,n,k", [(700, 900, 9001), (200, 1000, 20000), (355, 1296, 15040), (512, 512, 16390)])
def test_split_sums_on_two_streams_at_once(m, n, k):
    """Two products at once, each with a workspace of its own."""
    assert uq.uq_mx4_matmul_workspace_bytes(m, n, k) > 256  # k is split
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    work = []
    for i in range(2):
        rng = np.random.default_rng(m + i)
        a, b = operand(m, k, rng, 126, 128, 0), operand(n, k, rng, 126, 128, 0)
        ws = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
        work.append((a, b, ws, [new_out(m, n, "fp32") for _ in range(3)]))
    torch.cuda.synchronize()
    for j in range(3):
        for (a, b, ws, outs), side in zip(work, sides):
            with torch.cuda.stream(side):
                matmul(a, b, m, n, k, "fp32", outs[j], 0, ws)
    torch.cuda.synchronize()
    for a, b, _, outs in work:
        want = torch.from_numpy(a[2]) @ torch.from_numpy(b[2]).t()
        for out in outs:
            assert torch.equal(out[:, :n].cpu().double(), want)


@pytest.mark.parametrize("m,n,k", [(1, 300, 700), (40, 8200, 512), (300, 200, 4096), (700, 900, 9001), (300, 5001, 600),
                                   (998, 3709, 1993), (5001, 2003, 257), (3971, 4352, 262)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_replays(m, n, k, accumulate):
    """Captured once; the replays read the operands as they then are, between
    eager products on the same operands."""
    rng = np.random.default_rng(k)
    a, b = operand(m, k, rng, 126, 128, 0), operand(n, k, rng, 126, 128, 0)
    ws = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out, eager = new_out(m, n, "fp32"), new_out(m, n, "fp32")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        matmul(a, b, m, n, k, "fp32", out, accumulate, ws)
    b_values = torch.from_numpy(b[2]).t()
    want = torch.full((m, n), -3.0, dtype=torch.float64)
    for _ in range(4):
        fresh = operand(m, k, rng, 126, 128, 0)
        a[0].copy_(fresh[0])
        a[1].copy_(fresh[1])
        want = torch.from_numpy(fresh[2]) @ b_values + (want if accumulate else 0.0)
        graph.replay()
        matmul(a, b, m, n, k, "fp32", eager, accumulate)
        torch.cuda.synchronize()
        assert torch.equal(out[:, :n].cpu().double(), want)
        assert torch.equal(eager[:, :n].cpu().double(), want)
    assert (out[:, n:] == -3.0).all()


def test_one_matrix_as_both_operands():
    """x x^T from one set of codes."""
    a = operand(1270, 700, np.random.default_rng(2), 126, 128, 1)
    out = new_out(1270, 1270, "fp32")
    matmul(a, a, 1270, 1270, 700, "fp32", out, 0)
    torch.cuda.synchronize()
    v = torch.from_numpy(a[2])
    assert torch.equal(out[:, :1270].cpu().double(), v @ v.t())


def test_layer_that_grows_its_workspace_on_a_given_stream():
    """Fewer rows whose k is split need more workspace than the layer was made
    for; it is taken while the current stream is busy and the call goes to
    another one, given as a handle, then as a Stream, then as the default."""
    from oracle import mx4
    from paper_2109_12497_amd.mx4 import Mx4Linear

    tokens, rows, inputs, outputs = 4096, 512, 16384, 1000
    assert uq.uq_mx4_matmul_workspace_bytes(rows, outputs, inputs) > uq.uq_mx4_matmul_workspace_bytes(
        tokens, outputs, inputs)
    gen = torch.Generator().manual_seed(3)
    xh, wh = (torch.randint(-6, 7, (n, inputs), generator=gen).float() for n in (rows, outputs))
    x, w = xh.to(DEV), wh.to(DEV)
    busy = torch.randn(4096, 4096, device=DEV)

    def seen(v):
        codes, scales = mx4.quantize(v.numpy(), None)
        return torch.from_numpy(mx4.decode(codes, scales, inputs))

    want = seen(xh) @ seen(wh).t()  # multiples of 1 below 2^24
    side = torch.cuda.Stream()
    for stream in (side.cuda_stream, side, torch.cuda.default_stream(), None):
        layer = Mx4Linear(tokens, inputs, outputs, device=DEV, train=False)
        torch.cuda.synchronize()
        for _ in range(8):
            busy = torch.sin(busy)
        layer.load(w, stream=stream)
        y = layer.forward(x, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(y.cpu().double(), want)


@pytest.mark.parametrize("m,n,k,dtype", [(5901, 5703, 64, "fp32"), (8201, 8190, 40, "bf16"), (65537, 1030, 300, "fp16"),
                                         (33001, 1025, 65, "fp32")])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_outputs_that_pass_the_cache_by(m, n, k, dtype, accumulate):
    """128 MiB of outputs and more."""
    assert m * n * (4 if dtype == "fp32" else 2) >= 128 << 20
    out, want, _, _ = case(m, n, k, dtype, accumulate, m + n + k)
    assert torch.equal(out[:, :n].cpu(), want.to(out.dtype))
    assert (out[:, n:] == -3.0).all()
