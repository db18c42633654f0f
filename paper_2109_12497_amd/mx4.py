"""Microscaled 4-bit floating point through the C ABI: a linear layer whose
three products run on 4-bit operands, and the aggregation step on 4-bit codes.

Like `Step`, each class owns the device buffers of a fixed problem shape and
issues the library calls; no arithmetic of the method happens here.  Calls go
to the current stream of the device the buffers are on, or to the one given.
"""
from __future__ import annotations

import functools

import torch

from . import (UQ_BF16, UQ_F16, UQ_F32, _stream, uq_mx4_aggregate, uq_mx4_matmul, uq_mx4_matmul_workspace_bytes, uq_mx4_quantize,
               uq_mx4_quantize_sum, uq_mx4_shared_scale)
from .step import round_up

TYPES = {torch.float32: UQ_F32, torch.bfloat16: UQ_BF16, torch.float16: UQ_F16}


def _device(device) -> torch.device:
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    return device


def _settle(device) -> None:
    """Waits for the fills of new buffers, which the first call may use on
    another stream."""
    if device.type == "cuda" and not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream(device).synchronize()


@functools.lru_cache(maxsize=256)
def _layer_workspace_bytes(tokens: int, inputs: int, outputs: int, train: bool) -> int:
    """What the products of any number of rows up to `tokens` need at most.
    Fewer rows can need more: k is split where tiles are few.  (A plan takes
    about 1.5 us of the host, so 8192 tokens about 40 ms, once for a shape.)"""
    most = 0
    for rows in range(1, tokens + 1):
        most = max(most, uq_mx4_matmul_workspace_bytes(rows, outputs, inputs))
        if train:
            most = max(most, uq_mx4_matmul_workspace_bytes(rows, inputs, outputs),
                       uq_mx4_matmul_workspace_bytes(outputs, inputs, rows))
    return most


def _check_matrix(t, rows: int, cols: int, device) -> None:
    """A [rows, cols] matrix whose rows the calls can read in 16-byte pieces."""
    assert t.dtype in TYPES and t.device == device and tuple(t.shape) == (rows, cols)
    assert cols == 1 or t.stride(1) == 1
    # a call would go to another device's stream
    assert torch.cuda.current_device() == device.index, "the current device is not the buffers'"


def _ld(t) -> int:
    """The leading dimension: of a single row or an empty matrix any that fits."""
    mult = 4 if t.dtype == torch.float32 else 8
    return round_up(max(t.shape[1], 1), mult) if t.shape[0] <= 1 else t.stride(0)


class Codes:
    """Buffers of a rows x cols matrix held as codes and scale bytes."""

    def __init__(self, rows: int, cols: int, device):
        blocks = -(-cols // 32)
        self.codes = torch.zeros((rows, 16 * max(blocks, 1)), dtype=torch.uint8, device=device)
        self.scales = torch.zeros((rows, round_up(max(blocks, 1), 16)), dtype=torch.uint8, device=device)

    def args(self):
        return self.codes, self.codes.stride(0), self.scales, self.scales.stride(0)


def quantize(x, rows: Codes | None, cols: Codes | None, stochastic: bool = False, seed: int = 0, stream=None) -> None:
    """The codes of x along its rows and those of its transpose, or either."""
    none = (None, 0, None, 0)
    uq_mx4_quantize(x, TYPES[x.dtype], x.shape[0], x.shape[1], _ld(x), int(stochastic), seed,
                    *(none if rows is None else rows.args()), *(none if cols is None else cols.args()), stream)


class Mx4Linear:
    """y = x w^T, and in the backward pass dx = dy w and dw = dy^T x, each
    product of two matrices held as 4-bit codes whose blocks run along the
    summed dimension.

    load(w) quantises the weight [outputs, inputs] to the nearest, along both
    dimensions; a training program calls it after every update, a serving one
    once.  forward(x) takes up to `tokens` rows; with train=True it also keeps
    the transposed codes of x for dw.  backward(dy, seed) rounds dy
    stochastically, so that both gradients are without bias given the
    quantised x and w, and returns (dx, dw); with accumulate=True dw is added to
    what the buffer holds.  The uniform words are those of (seed, row, column)
    alone: every layer and every step needs a seed of its own (step * layers +
    layer, say), and so does a Mx4Step or Step on the gradients.  Where one seed
    rounds a layer's dy and then the dy formed from it, the second rounding
    depends on what it rounds and the chain is biased.  y, dx and dw are views of the layer's own buffers (y
    and dx of `dtype`, dw in binary32) and stay until the next call that
    writes them.  Rows of x, w and dy start on 16-byte boundaries, and the layer
    is called by hand: it takes no part in autograd.  Calls allocate nothing: the workspace is sized once, for the
    number of rows that needs the most.
    """

    def __init__(self, tokens: int, inputs: int, outputs: int, dtype=torch.float32, device="cuda", train: bool = True):
        assert dtype in TYPES and tokens >= 1 and inputs >= 1 and outputs >= 1
        self.tokens, self.inputs, self.outputs, self.dtype, self.train = tokens, inputs, outputs, dtype, train
        self.device = dev = _device(device)
        self.x = Codes(tokens, inputs, dev)
        self.w = Codes(outputs, inputs, dev)
        self.y = torch.zeros((tokens, round_up(outputs, 8)), dtype=dtype, device=dev)
        if train:
            self.x_t = Codes(inputs, tokens, dev)
            self.w_t = Codes(inputs, outputs, dev)
            self.dy = Codes(tokens, outputs, dev)
            self.dy_t = Codes(outputs, tokens, dev)
            self.dx = torch.zeros((tokens, round_up(inputs, 8)), dtype=dtype, device=dev)
            self.dw = torch.zeros((outputs, round_up(inputs, 4)), dtype=torch.float32, device=dev)
        # for every number of rows, so that no call allocates and a captured graph's stays where it is
        self.ws = torch.empty(_layer_workspace_bytes(tokens, inputs, outputs, train), dtype=torch.uint8, device=dev)
        self.rows = 0  # of the last forward
        _settle(dev)

    def _matmul(self, a: Codes, b: Codes, m: int, n: int, k: int, out, accumulate: bool, stream) -> None:
        uq_mx4_matmul(*a.args(), *b.args(), m, n, k, TYPES[out.dtype], out, out.stride(0), int(accumulate), self.ws,
                      self.ws.numel(), stream)

    def load(self, w, stream=None) -> None:
        _check_matrix(w, self.outputs, self.inputs, self.device)
        quantize(w, self.w, self.w_t if self.train else None, stream=_stream(stream))

    def forward(self, x, stream=None):
        """x [rows, inputs], rows <= tokens.  Returns the view y [rows, outputs]."""
        rows = x.shape[0]
        assert rows <= self.tokens
        _check_matrix(x, rows, self.inputs, self.device)
        stream = _stream(stream)  # resolved once for the calls
        self.rows = rows
        quantize(x, self.x, self.x_t if self.train else None, stream=stream)
        self._matmul(self.x, self.w, rows, self.outputs, self.inputs, self.y, False, stream)
        return self.y[:rows, :self.outputs]

    def backward(self, dy, seed: int, accumulate: bool = False, stream=None):
        """dy [rows, outputs] of the last forward's rows.  Returns the views
        (dx [rows, inputs], dw [outputs, inputs])."""
        assert self.train, "the layer keeps no transposed codes (train=False)"
        rows = dy.shape[0]
        assert rows == self.rows, "dy has not the rows of the last forward"
        _check_matrix(dy, rows, self.outputs, self.device)
        stream = _stream(stream)
        quantize(dy, self.dy, self.dy_t, stochastic=True, seed=seed, stream=stream)
        self._matmul(self.dy, self.w_t, rows, self.inputs, self.outputs, self.dx, False, stream)
        self._matmul(self.dy_t, self.x_t, self.outputs, self.inputs, rows, self.dw, accumulate, stream)
        return self.dx[:rows, :self.inputs], self.dw[:, :self.inputs]


class Mx4Step:
    """One aggregation step on 4-bit codes with shared scale bytes, for M
    workers' gradients g [M, ldg] fp32.

    run() is one library call for up to 16 resident rows (uq_mx4_aggregate).
    With streamed=True, or more rows, the shared bytes are formed first and the
    workers' codes then added to the resident sum: one worker at a time when
    streamed, else all at once; the same results, bit for bit.
    """

    def __init__(self, d: int, M: int, device="cuda", streamed: bool = False):
        assert d >= 0 and M >= 1
        self.d, self.M, self.streamed = d, M, streamed
        self.device = _device(device)
        self.scales = torch.zeros(round_up(max(-(-d // 32), 1), 16), dtype=torch.uint8, device=self.device)
        self.sum = torch.zeros(round_up(max(d, 1), 64), dtype=torch.int32, device=self.device)
        self.out = torch.zeros(round_up(max(d, 1), 64), dtype=torch.float32, device=self.device)
        _settle(self.device)

    def run(self, g, seed: int, stream=None):
        """g: [M, ldg] float32 on the device.  Returns the output view [d]."""
        assert g.dtype == torch.float32 and g.device == self.device and g.shape[0] == self.M
        assert g.stride(1) == 1 and g.shape[1] >= self.d
        assert torch.cuda.current_device() == self.device.index, "the current device is not the buffers'"
        d, M, ldg = self.d, self.M, g.stride(0)
        stream = _stream(stream)  # resolved once for the step's calls
        if not self.streamed and M <= 16:
            uq_mx4_aggregate(g, d, M, ldg, seed, self.scales, self.sum, self.out, stream)
            return self.out[:d]
        each = 1 if self.streamed else M
        for m in range(0, M, each):
            uq_mx4_shared_scale(g[m:m + each], d, each, ldg, int(m > 0), self.scales, stream)
        for m in range(0, M, each):
            uq_mx4_quantize_sum(g[m:m + each], d, each, ldg, m, self.scales, seed, int(m > 0), self.sum, M,
                                self.out if m + each == M else None, stream)
        return self.out[:d]
