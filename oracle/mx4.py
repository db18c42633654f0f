"""TEST INFRASTRUCTURE ONLY: microscaled 4-bit floating point in 64 bits.

A plain numpy implementation of the format, rounding rules, product and
aggregation step that include/uq.h defines, written from those definitions;
used only by the tests.
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
_LOW = np.uint64(0xFFFFFFFF)


def _blocks(cols: int) -> int:
    return -(-cols // 32)


def words(rows: int, cols: int, row0: int, seed: int) -> np.ndarray:
    """The 32-bit uniform words [rows, cols]: Philox4x32-10 blocks with
    counter (octet, row, 0) for the high and (octet, row, 1) for the low half."""
    octets = -(-cols // 8)
    octet, row = np.meshgrid(np.arange(octets, dtype=np.uint64), np.arange(row0, row0 + rows, dtype=np.uint64))
    out = np.zeros((rows, octets * 8), dtype=np.uint64)
    for last, shift in ((0, 16), (1, 0)):
        c = [octet & _LOW, octet >> np.uint64(32), row, np.full_like(row, last)]
        k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
        for _ in range(10):
            pa, pb = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(pb >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), pb & _LOW,
                 (pa >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), pa & _LOW]
            k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
        for h in range(8):
            half = (c[h % 4] >> np.uint64(16 * (h // 4))) & np.uint64(0xFFFF)
            out[:, h::8] |= half << np.uint64(shift)
    return out[:, :cols]


def block_max(x: np.ndarray) -> np.ndarray:
    """Largest |x| of each block, NaN where the block holds one."""
    r, c = x.shape
    full = np.zeros((r, _blocks(c) * 32))
    full[:, :c] = np.abs(x.astype(np.float64))
    return full.reshape(r, _blocks(c), 32).max(-1)


def bytes_of(top: np.ndarray) -> np.ndarray:
    """Scale bytes of block maxima: the least e >= -126 with top <= 6 * 2^e."""
    out = np.full(top.shape, 255, dtype=np.int64)
    fine = np.isfinite(top)
    e = np.full(top.shape, -126, dtype=np.int64)
    for step in range(-126, 127):
        e = np.where(fine & (top > 6.0 * 2.0 ** step), step + 1, e)
    out[fine] = e[fine] + 127
    return out.astype(np.uint8)


def fields(x: np.ndarray, scale_bytes: np.ndarray, r: np.ndarray | None) -> np.ndarray:
    """The 4-bit fields [rows, cols] of x on the given bytes; r: the elements'
    uniform words, or None for rounding to the nearest."""
    rows, c = x.shape
    b = np.repeat(scale_bytes.astype(np.int64), 32, axis=1)[:, :c]
    bad = b == 255
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.abs(x.astype(np.float64)) * 2.0 ** (127.0 - np.maximum(b, 1))
    y = np.where(bad, 0.0, y)
    y = np.where(np.isnan(y), 6.0, np.minimum(y, 6.0))
    at = np.clip(np.searchsorted(LEVELS, y, side="right") - 1, 0, 6)
    part = (y - LEVELS[at]) / (LEVELS[at + 1] - LEVELS[at])
    if r is None:
        up = (part > 0.5) | ((part == 0.5) & (at % 2 == 1))
    else:
        up = (r.astype(np.float64) < np.floor(part * 2.0 ** 32)) | (part == 1.0)
    code = at + up
    return np.where(bad, 0, code | (np.signbit(x).astype(np.int64) << 3)).astype(np.uint8)


def pack(f: np.ndarray) -> np.ndarray:
    """Fields [rows, cols] as bytes [rows, 16 * ceil(cols / 32)]."""
    r, c = f.shape
    full = np.zeros((r, _blocks(c) * 32), dtype=np.uint8)
    full[:, :c] = f
    return full[:, 0::2] | (full[:, 1::2] << 4)


def quantize(x: np.ndarray, r: np.ndarray | None):
    """(packed codes, scale bytes) of x."""
    b = bytes_of(block_max(x))
    return pack(fields(x, b, r)), b


def decode(codes: np.ndarray, scale_bytes: np.ndarray, cols: int) -> np.ndarray:
    """The values in 64 bits (NaN for byte 255)."""
    f = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], 2 * codes.shape[1])[:, :cols]
    v = np.where(f > 7, -1.0, 1.0) * LEVELS[f & 7]
    b = np.repeat(scale_bytes.astype(np.int64), 32, axis=1)[:, :cols]
    return np.where(b == 255, np.nan, v * 2.0 ** (np.where(b == 255, 0, b) - 127.0))


def quantize_sum(g: np.ndarray, d: int, scale_bytes: np.ndarray, seed: int, worker0: int = 0) -> np.ndarray:
    """The rows' codes in half units on shared bytes, added (int64 [d])."""
    rows = g.shape[0]
    b = np.broadcast_to(scale_bytes[None, :], (rows, scale_bytes.size))
    f = fields(g[:, :d], b, words(rows, d, worker0, seed))
    return (np.where(f > 7, -1, 1) * (2 * LEVELS[f & 7]).astype(np.int64)).sum(0)


def mean(total: np.ndarray, scale_bytes: np.ndarray, M: int) -> np.ndarray:
    """RN32(sum * 2^(e - 1) / M), NaN for byte 255: the quotient of integers below
    2^31 in 64 bits, which rounds to the binary32 number that the exact one does."""
    b = np.repeat(scale_bytes.astype(np.int64), 32)[:total.size]
    half = 2.0 ** (np.where((b == 255) | (b < 1), 1, b) - 128.0)
    with np.errstate(over="ignore"):
        out = (total.astype(np.float64) / M * half).astype(np.float32)
    return np.where(b == 255, np.float32(np.nan), out).astype(np.float32)


def aggregate(g: np.ndarray, d: int, seed: int):
    """(bytes, sum, out) of the whole step over the rows of g."""
    b = bytes_of(block_max(g[:, :d])).max(0) if d else np.zeros(0, dtype=np.uint8)
    s = quantize_sum(g, d, b, seed)
    return b, s, mean(s, b, g.shape[0])
