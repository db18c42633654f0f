"""The aggregation step on microscaled 4-bit codes, bit for bit against the
64-bit implementation, in its one-call and its separate forms."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2109_12497_amd as uq  # noqa: E402
import synth  # noqa: E402
from oracle import mx4  # noqa: E402

DEV = torch.device("cuda:0")
PAD = 64


def buffers(d):
    return (torch.full((-(-d // 32) + PAD,), 0xA5, dtype=torch.uint8, device=DEV),
            torch.full((d + PAD,), -77, dtype=torch.int32, device=DEV),
            torch.full((d + PAD,), -7.0, dtype=torch.float32, device=DEV))


def untouched(bufs, d):
    s, t, o = bufs
    assert (s[-(-d // 32):] == 0xA5).all() and (t[d:] == -77).all() and (o[d:] == -7.0).all()


def equal_bits(got, want):
    a, b = got.cpu().numpy(), want
    assert np.array_equal(np.isnan(a), np.isnan(b))
    fine = ~np.isnan(b)
    assert np.array_equal(a[fine].view(np.int32), b[fine].view(np.int32))


def gradients(M, d, seed):
    host = synth.mixed_rows(M, d, seed=seed, ldg=synth.round_up(d, 64) + 64)
    host[:, d:] = np.nan  # never read into a result
    return host


@pytest.mark.parametrize("d", [1, 7, 31, 32, 33, 63, 100, 1000, 2048, 4097, 10_007, 300_001])
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 8, 9, 12, 13, 16])
def test_one_call(d, M):
    host = gradients(M, d, d + M)
    seed = 0xABCDEF0123 + d
    bufs = s, t, o = buffers(d)
    uq.uq_mx4_aggregate(torch.from_numpy(host).to(DEV), d, M, host.shape[1], seed, s, t, o)
    torch.cuda.synchronize()
    b, total, out = mx4.aggregate(host, d, seed)
    assert np.array_equal(s[:b.size].cpu().numpy(), b)
    assert np.array_equal(t[:d].cpu().numpy(), total)
    equal_bits(o[:d], out)
    untouched(bufs, d)


@pytest.mark.parametrize("d,M,groups", [(1000, 5, (1, 1, 1, 1, 1)), (10_007, 20, (7, 13)), (2_049, 3, (3,)), (33, 40, (40,)),
                                        (70_001, 17, (16, 1))])
def test_separate_calls(d, M, groups):
    """Any grouping of the workers gives the bytes, sums and means of all."""
    host = gradients(M, d, M)
    g = torch.from_numpy(host).to(DEV)
    bufs = s, t, o = buffers(d)
    first = 0
    for n in groups:
        uq.uq_mx4_shared_scale(g[first:first + n], d, n, host.shape[1], int(first > 0), s)
        first += n
    first = 0
    for n in groups:
        uq.uq_mx4_quantize_sum(g[first:first + n], d, n, host.shape[1], first, s, 4242, int(first > 0), t, M,
                               o if first + n == M else None)
        first += n
    torch.cuda.synchronize()
    b, total, out = mx4.aggregate(host, d, 4242)
    assert np.array_equal(s[:b.size].cpu().numpy(), b)
    assert np.array_equal(t[:d].cpu().numpy(), total)
    equal_bits(o[:d], out)
    untouched(bufs, d)


def special_rows(M):
    """Blocks of zeros, of extremes, of denormals, and of one worker's NaN or infinity."""
    d = 32 * 12
    rng = np.random.default_rng(1)
    host = rng.normal(size=(M, d)).astype(np.float32)
    host[:, 0:32] = 0.0
    host[:, 32:64] = -0.0
    with np.errstate(over="ignore"):  # some workers' products reach infinity
        host[:, 64:96] *= np.float32(1.5e38)
    host[0, 64] = np.finfo(np.float32).max
    host[:, 96:128] *= np.float32(1e-42)
    host[1, 130] = np.nan
    host[M - 1, 170] = np.inf
    host[0, 200] = -np.inf
    host[:, 224:256] *= np.float32(2.0 ** -126)
    host[1, 256:288] *= np.float32(1e20)  # the others fall far below its grid
    host[:, 288:320] = np.tile(np.array([0, 1, 2, 3, 4, 6, 8, 12], dtype=np.float32) * 0.5, 4)
    return host, d


@pytest.mark.parametrize("M", [2, 7, 16])
def test_special_values(M):
    host, d = special_rows(M)
    g = torch.from_numpy(host).to(DEV)
    bufs = s, t, o = buffers(d)
    uq.uq_mx4_aggregate(g, d, M, d, 3, s, t, o)
    torch.cuda.synchronize()
    b, total, out = mx4.aggregate(host, d, 3)
    assert (b[4:7] == 255).all() and (b[[0, 1, 3, 7, 8, 9, 10, 11]] != 255).all()
    assert np.array_equal(s[:b.size].cpu().numpy(), b)
    assert np.array_equal(t[:d].cpu().numpy(), total)
    equal_bits(o[:d], out)
    bufs2 = s2, t2, o2 = buffers(d)
    uq.uq_mx4_shared_scale(g, d, M, d, 0, s2)
    uq.uq_mx4_quantize_sum(g, d, M, d, 0, s2, 3, 0, t2, M, o2)
    torch.cuda.synchronize()
    assert torch.equal(s, s2) and torch.equal(t, t2)
    equal_bits(o2[:d], out)


def test_bytes_smaller_than_needed_saturate():
    """Shared bytes that do not cover a row: magnitudes beyond take code 7, a
    byte of 0 is read as 1, one of 254 holds the codes it stands for."""
    d = 32 * 6
    rng = np.random.default_rng(2)
    host = rng.normal(size=(3, d)).astype(np.float32)
    host[0, 5], host[1, 70], host[2, 100] = np.inf, np.nan, -np.inf
    b = np.array([125, 100, 0, 254, 1, 127], dtype=np.uint8)
    s, t, o = buffers(d)
    s[:6] = torch.from_numpy(b).to(DEV)
    uq.uq_mx4_quantize_sum(torch.from_numpy(host).to(DEV), d, 3, d, 0, s, 8, 0, t, 3, o)
    torch.cuda.synchronize()
    total = mx4.quantize_sum(host, d, b, 8)
    assert np.array_equal(t[:d].cpu().numpy(), total)
    assert np.array_equal(s[:6].cpu().numpy(), b)


def test_ties_of_the_high_half():
    """Elements made from the uniform words, so that the low halves decide."""
    M, d, seed = 4, 32 * 64, 21
    r = mx4.words(M, d, 0, seed)
    for base, step in ((0.0, 0.5), (1.5, 0.5), (3.0, 1.0), (4.0, 2.0)):
        host = (base + step * ((r >> np.uint64(16)).astype(np.float64) + 0.5) / 65536.0).astype(np.float32)
        host[:, ::32] = 6.0
        s, t, o = buffers(d)
        uq.uq_mx4_aggregate(torch.from_numpy(host).to(DEV), d, M, d, seed, s, t, o)
        torch.cuda.synchronize()
        b, total, out = mx4.aggregate(host, d, seed)
        assert np.array_equal(t[:d].cpu().numpy(), total)
        equal_bits(o[:d], out)


def test_capped_grid():
    M, d = 6, 90_001
    host = gradients(M, d, 5)
    g = torch.from_numpy(host).to(DEV)
    s, t, o = buffers(d)
    s2, t2, o2 = buffers(d)
    uq.uq_set_grid_cap(8)
    try:
        uq.uq_mx4_aggregate(g, d, M, host.shape[1], 6, s, t, o)
        uq.uq_mx4_shared_scale(g, d, M, host.shape[1], 0, s2)
        uq.uq_mx4_quantize_sum(g, d, M, host.shape[1], 0, s2, 6, 0, t2, M, o2)
    finally:
        uq.uq_set_grid_cap(0)
    torch.cuda.synchronize()
    b, total, out = mx4.aggregate(host, d, 6)
    assert np.array_equal(s[:b.size].cpu().numpy(), b) and torch.equal(s, s2)
    assert np.array_equal(t[:d].cpu().numpy(), total) and torch.equal(t, t2)
    equal_bits(o[:d], out)
    equal_bits(o2[:d], out)


def test_offsets_past_2_to_31():
    """Two rows of 1.1 G coordinates (byte offsets past 2^32), checked where
    the offsets wrap and at the end."""
    M, d = 2, 1_100_000_033
    ldg = synth.round_up(d, 64)
    g = torch.empty((M, ldg), dtype=torch.float32, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(4)
    for m in range(M):
        g[m].normal_(generator=gen)
    s, t, o = buffers(d)
    uq.uq_mx4_aggregate(g, d, M, ldg, 12, s, t, o)
    torch.cuda.synchronize()
    for i0 in (0, (1 << 29) - 64, (1 << 30) - 32, d // 32 * 32 - 96):
        i1 = min(d, i0 + 128)
        sub = g[:, i0:i1].cpu().numpy()
        b = mx4.bytes_of(mx4.block_max(sub)).max(0)
        assert np.array_equal(s[i0 // 32:i0 // 32 + b.size].cpu().numpy(), b)
        words = [np.array([O_word(12, m, i) for i in range(i0, i1)], dtype=np.uint64) for m in range(M)]
        f = mx4.fields(sub, np.tile(b, (M, 1)), np.stack(words))
        total = (np.where(f > 7, -1, 1) * (2 * mx4.LEVELS[f & 7]).astype(np.int64)).sum(0)
        assert np.array_equal(t[i0:i1].cpu().numpy(), total)
        equal_bits(o[i0:i1], mx4.mean(total, b, M))


def O_word(seed, worker, i):
    from oracle import oracle

    return oracle.uniform_word(seed, worker, i)
