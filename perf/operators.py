"""Timed cases of the microscaled 4-bit floating-point operators.

The format: a row's elements in blocks of 32; each block has one scale byte
(2^(byte - 127), 255: NaN) and 32 fields of 4 bits, the element's sign above a
code 0..7 for the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4 and 6.

A case's fields:
  op      "round trip"  quantise a matrix and read the result back: the codes of
                        the rows, of the transposed matrix, or of both
          "read"        the values of codes that a program holds
          "product"     out[i][j] (+)= sum_k a[i][k] b[j][k] of quantised a, b
          "step"        M workers' gradients averaged through codes on shared
                        scales, in one call
          "streamed"    the same with the workers one after another
  dtype   of the matrix, and of what is read back, or of the product's output
  "round trip": rows, cols, form ("rows", "transposed", "both"), stochastic
  "read":       rows, cols
  "product":    m, n, k, accumulate
  "step", "streamed": d, M
  pad     extra elements between rows (16-byte multiples)

Listed cases, and what each stands for:
  token-round-trip     one token's activations, where latency is all the time there is
  ragged-round-trip    odd sizes, stochastic, both orientations
  train-round-trip     an output gradient of a training step: the operands of both
                       products of the backward pass from one read
  ragged-read, large-read  weights kept in 4 bits, read back
  token-product        one token through a layer: the weights are read once
  few-rows-product     a few dozen tokens, odd sizes throughout
  grad-product         a weight gradient added to its fp32 accumulator
  large-product        a training layer's forward product
  sgd-step             the convergence demo's gradient, 1000 coordinates, 8 workers
  resnet50-step        ResNet-50 gradients, 8 workers resident
  vgg16-streamed       VGG-16 gradients, 4 workers, one after another
`draw` spreads the same operators over sizes, types, forms and strides.
"""
from __future__ import annotations

import math

import torch

own = False

RESNET50, VGG16 = 25_557_032, 138_357_544
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
TYPE_IDS = {"fp32": 0, "bf16": 1, "fp16": 2}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _round_trip(rows, cols, dtype, form, stochastic, pad=0, **kw):
    return dict(op="round trip", rows=rows, cols=cols, dtype=dtype, form=form, stochastic=stochastic, pad=pad, **kw)


def _read(rows, cols, dtype, pad=0, **kw):
    return dict(op="read", rows=rows, cols=cols, dtype=dtype, pad=pad, **kw)


def _product(m, n, k, dtype, accumulate, pad=0, **kw):
    return dict(op="product", m=m, n=n, k=k, dtype=dtype, accumulate=accumulate, pad=pad, **kw)


def _step(op, d, M, **kw):
    return dict(op=op, d=d, M=M, dtype="fp32", **kw)


def listed():
    return [
        _round_trip(1, 4096, "bf16", "rows", False, name="token-round-trip"),
        _round_trip(1021, 5003, "fp16", "both", True, pad=24, name="ragged-round-trip"),
        _round_trip(8192, 8192, "bf16", "both", True, name="train-round-trip"),
        _read(1021, 1531, "fp16", pad=8, name="ragged-read"),
        _read(16384, 8192, "bf16", name="large-read"),
        _product(1, 8192, 8192, "bf16", False, name="token-product"),
        _product(37, 10_001, 5003, "fp32", False, pad=16, name="few-rows-product"),
        _product(4096, 4096, 8192, "fp32", True, name="grad-product"),
        _product(8192, 8192, 8192, "bf16", False, name="large-product"),
        _step("step", 1000, 8, name="sgd-step"),
        _step("step", RESNET50, 8, name="resnet50-step"),
        _step("streamed", VGG16, 4, name="vgg16-streamed"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def size(lo, hi):
        n = log_int(lo, hi)
        if n > 64 and rng.random() < 0.4:
            n = min(hi, -(-n // 64) * 64)
        return n

    op = rng.choice(["round trip", "round trip", "read", "product", "product", "product", "step", "streamed"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    pad = rng.choice([0, 0, 8, 64])
    if op in ("round trip", "read"):
        rows, cols = size(1, 16384), size(8, 16384)
        rows = max(1, min(rows, 8192 * 8192 // cols))
        if op == "read":
            return _read(rows, cols, dtype, pad)
        return _round_trip(rows, cols, dtype, rng.choice(["rows", "transposed", "both"]), rng.random() < 0.5, pad)
    if op == "product":
        m, n, k = size(1, 8192), size(8, 16384), size(32, 16384)
        m = max(1, min(m, 8192 ** 3 // (n * k)))
        return _product(m, n, k, dtype, rng.random() < 0.4, rng.choice([0, 16, 64]))
    M = rng.randint(1, 16)
    d = min(log_int(1000, VGG16), 4 * VGG16 // M)
    if rng.random() < 0.5:
        d |= 1
    return _step(op, d, M)


# ---------------------------------------------------------------------------
# The plain forms.
# ---------------------------------------------------------------------------
_LOW = 0xFFFFFFFF


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 over int64 tensors that hold 32-bit words."""
    k0, k1 = seed & _LOW, (seed >> 32) & _LOW
    for _ in range(10):
        pa, pb = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (((pb >> 32) & _LOW) ^ c1 ^ k0, pb & _LOW, ((pa >> 32) & _LOW) ^ c3 ^ k1, pa & _LOW)
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return c0, c1, c2, c3


def _halves(row, octet, purpose, seed):
    """The eight 16-bit halves of each Philox block, [rows, 8 * octets]."""
    zero = torch.zeros_like(row + octet)
    words = torch.stack(_philox(zero + octet, zero, zero + row, zero + purpose, seed), dim=-1)
    return torch.cat([words & 0xFFFF, words >> 16], dim=-1).flatten(1)


def _uniforms(rows, cols, row0, seed):
    """The 32-bit uniform word of each element."""
    row = torch.arange(row0, row0 + rows, device="cuda", dtype=torch.int64)[:, None]
    octet = torch.arange(-(-cols // 8), device="cuda", dtype=torch.int64)[None, :]
    return ((_halves(row, octet, 0, seed) << 16) | _halves(row, octet, 1, seed))[:, :cols]


def _blocks(x):
    """|x| in 32 bits as [rows, blocks, 32], the last block filled with zeros."""
    r, c = x.shape
    mag = torch.zeros(r, -(-c // 32) * 32, dtype=torch.float32, device=x.device)
    mag[:, :c] = x.float().abs()
    return mag.view(r, -1, 32)


def _exponents(mag):
    """The least e >= -126 with max <= 6 * 2^e of each block, and 128 for a
    block that holds an infinity or a NaN."""
    top = mag.amax(-1)
    frac, p = torch.frexp(top)
    e = torch.where(frac <= 0.75, p - 3, p - 2).clamp(min=-126)
    e = torch.where(top == 0, torch.full_like(e, -126), e)
    return torch.where(torch.isfinite(top), e, torch.full_like(e, 128))


def _magnitudes(mag, e, words=None):
    """The codes' magnitudes in half units, as 32-bit floats [rows, blocks, 32]:
    rounded to the nearest, or by each element's uniform word."""
    fine = e < 128
    down = ((127 - torch.where(fine, e, 0)) << 23).to(torch.int32).view(torch.float32)  # 2^-e, by its bits
    y = torch.where(fine[..., None], mag * down[..., None], 0.0)
    step = torch.where(y < 2, 1.0, torch.where(y < 4, 2.0, 4.0))  # of the grid at y, in half units
    q = 2 * y / step
    if words is None:
        return torch.round(q) * step
    low = q.floor()
    t = ((q - low) * 4294967296.0).to(torch.int64)
    r = torch.zeros(mag.shape[0], mag.shape[1] * 32, dtype=torch.int64, device=mag.device)
    r[:, :words.shape[1]] = words
    return (low + (r.view(mag.shape) < t)) * step


def _power(e):
    """2^e in 64 bits, NaN for the exponent 128 of the scale byte 255."""
    two = ((e.to(torch.int64) + 1023) << 52).view(torch.float64)  # by its bits
    return torch.where(e < 128, two, math.nan)


def _plain_values(x, words):
    """What the codes of x stand for, in x's type."""
    mag = _blocks(x)
    e = _exponents(mag)
    half = _magnitudes(mag, e, words)
    v = (half.double() * (_power(e) / 2)[..., None]).flatten(1)[:, :x.shape[1]]
    return torch.copysign(v, x.double()).to(x.dtype)


def _plain_read(codes, scales, cols):
    """The values of packed codes in 32 bits."""
    field = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1)[:, :cols].to(torch.int32)
    c = field & 7
    mag = torch.where(c < 2, c, torch.where(c < 6, (2 + (c & 1)) * (c >> 1), 8 + 4 * (c & 1))) * 0.5
    power = _power(scales[:, :-(-cols // 32)].to(torch.int32) - 127)
    v = mag.double() * power.repeat_interleave(32, dim=1)[:, :cols]
    return torch.where(field > 7, -v, v).float()


def _plain_sum(g, e, seed, worker0):
    """The rows' codes in half units on the shared exponents e, added."""
    mag = _blocks(g)
    words = _uniforms(g.shape[0], g.shape[1], worker0, seed)
    half = _magnitudes(mag, e.expand(g.shape[0], -1), words).flatten(1)[:, :g.shape[1]]
    return torch.copysign(half, g).sum(0).to(torch.int32)


def _plain_step(g, seed):
    M, d = g.shape
    e = torch.full((1, -(-d // 32)), -126, dtype=torch.int32, device=g.device)
    for m in range(M):
        e = torch.maximum(e, _exponents(_blocks(g[m:m + 1])))
    total = torch.zeros(d, dtype=torch.int32, device=g.device)
    for m in range(M):
        total += _plain_sum(g[m:m + 1], e, seed, m)
    power = _power(e[0]).repeat_interleave(32)[:d]
    out = (total.double() * (power / (2 * M))).float()
    return dict(out=out, sum=total, scales=(torch.where(e[0] < 128, e[0], 128) + 127).to(torch.uint8))


# ---------------------------------------------------------------------------
# Inputs.
# ---------------------------------------------------------------------------
def _up(n, m):
    return -(-n // m) * m


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _matrix(rows, cols, dtype, pad, seed):
    """Normal values whose width differs from row to row and from column to
    column, with a few columns ten times wider, as activations have them."""
    gen = _generator(seed)
    ld = _up(cols, 8) + pad
    x = torch.empty(rows, ld, dtype=torch.float32, device="cuda").normal_(generator=gen)
    x *= torch.exp2(torch.empty(rows, 1, device="cuda").uniform_(-4, 2, generator=gen))
    wide = torch.rand(1, ld, device="cuda", generator=gen) < 0.01
    x *= torch.exp2(torch.empty(1, ld, device="cuda").uniform_(-2, 1, generator=gen)) * torch.where(wide, 10.0, 1.0)
    return x.to(DTYPES[dtype])


def _code_buffers(rows, cols, pad=0):
    """Codes and scale bytes of a rows x cols matrix, rows on 16-byte boundaries."""
    codes = torch.zeros(rows, 16 * -(-cols // 32) + pad, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(rows, _up(-(-cols // 32), 16) + pad, dtype=torch.uint8, device="cuda")
    return codes, scales


def _codes_of(x, codes, scales):
    """Nearest codes of x, packed (how a program's stored operands come about)."""
    cols = x.shape[1]
    mag = _blocks(x)
    e = _exponents(mag)
    half = _magnitudes(mag, e).flatten(1)
    c = torch.where(half < 4, half, torch.where(half < 8, 2 + half / 2, 4 + half / 4)).to(torch.uint8)
    c[:, :cols] |= torch.signbit(x).to(torch.uint8) << 3
    nb = e.shape[1]
    codes[:, :16 * nb] = c[:, 0::2] | (c[:, 1::2] << 4)
    scales[:, :nb] = (e + 127).to(torch.uint8)


def _gradients(case, seed):
    """The workers' gradients: 64 blocks of coordinates whose widths spread over three decades."""
    d, M = case["d"], case["M"]
    gen = _generator(seed)
    widths = 10.0 ** torch.empty(64, device="cuda").uniform_(-5, -2, generator=gen)
    g = torch.zeros(M, _up(d, 64), dtype=torch.float32, device="cuda")
    g[:, :d].normal_(generator=gen)
    g[:, :d] *= widths.repeat_interleave(-(-d // 64))[:d]
    return g


def _operands(case, seed):
    m, n, k, pad = case["m"], case["n"], case["k"], case["pad"]
    state = {}
    for name, rows, s in (("a", m, 1), ("b", n, 2)):
        codes, scales = _code_buffers(rows, k, pad)
        _codes_of(_matrix(rows, k, "bf16", 0, seed * 3 + s)[:, :k], codes, scales)
        state[name], state[name + "_scales"] = codes, scales
    out = torch.zeros(m, _up(n, 8) + pad, dtype=DTYPES[case["dtype"]], device="cuda")
    if case["accumulate"]:
        out.normal_(generator=_generator(seed * 3))
        out *= math.sqrt(k)
    state["out"] = out
    return state


def prepare(case, seed):
    op = case["op"]
    state = dict(case=case, seed=seed * 7919 + 1)
    if op == "round trip":
        rows, cols, pad, dt = case["rows"], case["cols"], case["pad"], DTYPES[case["dtype"]]
        state["x"] = _matrix(rows, cols, case["dtype"], pad, seed)
        state["codes"], state["scales"] = _code_buffers(rows, cols)
        state["codes_t"], state["scales_t"] = _code_buffers(cols, rows)
        state["values"] = torch.empty(rows, _up(cols, 8), dtype=dt, device="cuda")
        state["values_t"] = torch.empty(cols, _up(rows, 8), dtype=dt, device="cuda")
    elif op == "read":
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        state["codes"], state["scales"] = _code_buffers(rows, cols, 2 * pad)
        _codes_of(_matrix(rows, cols, "bf16", 0, seed)[:, :cols], state["codes"], state["scales"])
        state["values"] = torch.empty(rows, _up(cols, 8) + pad, dtype=DTYPES[case["dtype"]], device="cuda")
    elif op == "product":
        state.update(_operands(case, seed))
    else:
        d = case["d"]
        state["g"] = _gradients(case, seed)
        state["scales"] = torch.zeros(_up(-(-d // 32), 16), dtype=torch.uint8, device="cuda")
        state["sum"] = torch.zeros(_up(d, 64), dtype=torch.int32, device="cuda")
        state["out"] = torch.zeros(_up(d, 64), dtype=torch.float32, device="cuda")
    return state


# ---------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------
def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2109_12497_amd as uq

        return _OWN[op](uq, state, case, TYPE_IDS[case["dtype"]])
    if op == "round trip":
        x = state["x"][:, :case["cols"]]
        words = _uniforms(case["rows"], case["cols"], 0, state["seed"]) if case["stochastic"] else None
        res = {}
        if case["form"] != "transposed":
            res["values"] = _plain_values(x, words)
        if case["form"] != "rows":
            res["values_t"] = _plain_values(x.t(), None if words is None else words.t())
        return res
    if op == "read":
        return dict(values=_plain_read(state["codes"], state["scales"], case["cols"]).to(DTYPES[case["dtype"]]))
    if op == "product":
        a = _plain_read(state["a"], state["a_scales"], case["k"])
        b = _plain_read(state["b"], state["b_scales"], case["k"])
        out = state["out"][:, :case["n"]]
        p = a @ b.t()
        out.copy_(out.float() + p if case["accumulate"] else p)
        return dict(out=out)
    return _plain_step(state["g"][:, :case["d"]], state["seed"])


def _own_round_trip(uq, s, case, type_id):
    rows, cols, x = case["rows"], case["cols"], s["x"]
    by_rows, by_cols = case["form"] != "transposed", case["form"] != "rows"
    codes, scales = (s["codes"], s["scales"]) if by_rows else (None, None)
    codes_t, scales_t = (s["codes_t"], s["scales_t"]) if by_cols else (None, None)
    uq.uq_mx4_quantize(x, type_id, rows, cols, x.stride(0), int(case["stochastic"]), s["seed"],
                       codes, s["codes"].stride(0), scales, s["scales"].stride(0),
                       codes_t, s["codes_t"].stride(0), scales_t, s["scales_t"].stride(0))
    res = {}
    if by_rows:
        uq.uq_mx4_dequantize(codes, codes.stride(0), scales, scales.stride(0), rows, cols, type_id, s["values"],
                             s["values"].stride(0))
        res["values"] = s["values"][:, :cols]
    if by_cols:
        uq.uq_mx4_dequantize(codes_t, codes_t.stride(0), scales_t, scales_t.stride(0), cols, rows, type_id,
                             s["values_t"], s["values_t"].stride(0))
        res["values_t"] = s["values_t"][:, :rows]
    return res


def _own_read(uq, s, case, type_id):
    codes, scales, v = s["codes"], s["scales"], s["values"]
    uq.uq_mx4_dequantize(codes, codes.stride(0), scales, scales.stride(0), case["rows"], case["cols"], type_id, v,
                         v.stride(0))
    return dict(values=v[:, :case["cols"]])


def _own_product(uq, s, case, type_id):
    m, n, k, out = case["m"], case["n"], case["k"], s["out"]
    if "ws" not in s:  # kept by the program, as its other buffers
        s["ws"] = torch.empty(uq.uq_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda")
    uq.uq_mx4_matmul(s["a"], s["a"].stride(0), s["a_scales"], s["a_scales"].stride(0),
                     s["b"], s["b"].stride(0), s["b_scales"], s["b_scales"].stride(0),
                     m, n, k, type_id, out, out.stride(0), int(case["accumulate"]), s["ws"], s["ws"].numel())
    return dict(out=out[:, :n])


def _own_result(s, d):
    return dict(out=s["out"][:d], sum=s["sum"][:d], scales=s["scales"][:-(-d // 32)])


def _own_step(uq, s, case, type_id):
    d, M, g = case["d"], case["M"], s["g"]
    uq.uq_mx4_aggregate(g, d, M, g.stride(0), s["seed"], s["scales"], s["sum"], s["out"])
    return _own_result(s, d)


def _own_streamed(uq, s, case, type_id):
    d, M, g = case["d"], case["M"], s["g"]
    for m in range(M):
        uq.uq_mx4_shared_scale(g[m:m + 1], d, 1, g.stride(0), int(m > 0), s["scales"])
    for m in range(M):
        uq.uq_mx4_quantize_sum(g[m:m + 1], d, 1, g.stride(0), m, s["scales"], s["seed"], int(m > 0), s["sum"], M,
                               s["out"] if m == M - 1 else None)
    return _own_result(s, d)


_OWN = {"round trip": _own_round_trip, "read": _own_read, "product": _own_product, "step": _own_step,
        "streamed": _own_streamed}


def work(case):
    """Each input read once, each output written once; for a round trip also
    the codes, which are an output of its first half and the input of its second."""
    op, size = case["op"], SIZES[case["dtype"]]
    if op in ("round trip", "read"):
        n = case["rows"] * case["cols"]
        if op == "read":
            return {"bytes": n * 17 / 32 + size * n, "flops": n}
        ways = 2 if case["form"] == "both" else 1
        return {"bytes": size * n + ways * (2 * n * 17 / 32 + size * n), "flops": 2 * ways * n}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        outs = m * n * size * (2 if case["accumulate"] else 1)
        return {"bytes": (m + n) * k * 17 / 32 + outs, "flops": 2 * m * n * k}
    return {"bytes": 4 * case["M"] * case["d"] + 8 * case["d"] + case["d"] / 32, "flops": case["M"] * case["d"]}


# ---------------------------------------------------------------------------
# The same from the definition, in 64 bits.
# ---------------------------------------------------------------------------
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mul_words(a, b):
    """High and low words of the product of 32-bit words a (tensor) and b (number), by 16-bit halves."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    low, mid = a0 * b0, a0 * b1
    mid2 = a1 * b0 + mid + (low >> 16)
    return a1 * b1 + (mid2 >> 16), (low & 0xFFFF) | ((mid2 & 0xFFFF) << 16)


def _exact_words(rows, cols, row0, seed):
    """The uniform word of each element: block (octet, row) for the high half, with
    the last counter word 1 for the low half."""
    octets = -(-cols // 8)
    flat = torch.arange(rows * octets, device="cuda", dtype=torch.int64)
    words = 0
    for purpose, shift in ((0, 16), (1, 0)):
        x = [flat % octets, torch.zeros_like(flat), flat // octets + row0, torch.full_like(flat, purpose)]
        for i in range(10):
            k0 = ((seed & _LOW) + i * 0x9E3779B9) & _LOW
            k1 = ((seed >> 32) + i * 0xBB67AE85) & _LOW
            ha, la = _mul_words(x[0], 0xD2511F53)
            hb, lb = _mul_words(x[2], 0xCD9E8D57)
            x = [hb ^ x[1] ^ k0, lb, ha ^ x[3] ^ k1, la]
        eight = [(x[h % 4] >> (16 * (h // 4))) & 0xFFFF for h in range(8)]
        words = words | (torch.stack(eight, dim=1).view(rows, octets * 8)[:, :cols] << shift)
    return words


def _exact_power(e):
    table = torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device=e.device)
    return table[(e + 200).long()]


def _exact_scale(x):
    """The least e >= -126 with the block's largest magnitude at most 6 * 2^e (finite inputs)."""
    r, c = x.shape
    nb = -(-c // 32)
    full = torch.zeros(r, nb * 32, dtype=torch.float64, device=x.device)
    full[:, :c] = x.double().abs()
    top = full.view(r, nb, 32).max(-1).values
    e = torch.ceil(torch.log2(top / 6)).clamp(min=-126)
    e = e + (top > 6 * _exact_power(e)).double()
    return e - ((top <= 6 * _exact_power(e - 1)) & (e > -126)).double()


def _exact_round(x, e, words=None):
    """The values that the codes of x stand for on the exponents e, in 64 bits."""
    r, c = x.shape
    two = _exact_power(e).repeat_interleave(32, dim=1)[:, :c]
    y = x.double().abs() / two
    table = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    at = (torch.searchsorted(table, y, right=True) - 1).clamp(max=6)
    lo, hi = table[at], table[at + 1]
    part = (y - lo) / (hi - lo)
    if words is not None:
        up = words < torch.floor(part * 4294967296.0).to(torch.int64)
        up |= part >= 1
    else:
        up = (part > 0.5) | ((part == 0.5) & (at % 2 == 1))
    return torch.sign(x.double()) * torch.where(up, hi, lo) * two


def _exact_decode(codes, scales, cols):
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device=codes.device)
    v = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    v[:, 0::2] = table[(codes % 16).long()]
    v[:, 1::2] = table[(codes // 16).long()]
    at = torch.arange(cols, device=codes.device) // 32
    return v[:, :cols] * _exact_power(scales.double() - 127)[:, at]


def exact(case, seed):
    op, philox_seed = case["op"], seed * 7919 + 1
    if op == "round trip":
        x = _matrix(case["rows"], case["cols"], case["dtype"], case["pad"], seed)[:, :case["cols"]]
        words = _exact_words(case["rows"], case["cols"], 0, philox_seed) if case["stochastic"] else None
        res = {}
        if case["form"] != "transposed":
            res["values"] = _exact_round(x, _exact_scale(x), words)
        if case["form"] != "rows":
            x = x.t().contiguous()
            res["values_t"] = _exact_round(x, _exact_scale(x), None if words is None else words.t())
        return res
    if op == "read":
        state = prepare(case, seed)
        return dict(values=_exact_decode(state["codes"], state["scales"], case["cols"]))
    if op == "product":
        s = _operands(case, seed)
        a = _exact_decode(s["a"], s["a_scales"], case["k"])
        b = _exact_decode(s["b"], s["b_scales"], case["k"])
        p = a @ b.t()
        return dict(out=p + s["out"][:, :case["n"]].double() if case["accumulate"] else p)
    d, M = case["d"], case["M"]
    g = _gradients(case, seed)[:, :d]
    e = _exact_scale(g[:1])
    for m in range(1, M):
        e = torch.maximum(e, _exact_scale(g[m:m + 1]))
    total = torch.zeros(d, dtype=torch.float64, device="cuda")
    for m in range(M):
        total += _exact_round(g[m:m + 1], e, _exact_words(1, d, m, philox_seed))[0]
    return dict(out=total / M, sum=None, scales=None)
