"""The refusals of the microscaled 4-bit calls, checked without a GPU: every
invalid argument returns its status before anything touches the HIP runtime."""
import pytest

uq = pytest.importorskip("paper_2109_12497_amd", reason="libuq.so not built")
L = uq.lib

A = 0x10000  # a 16-byte aligned stand-in address; never dereferenced by a rejected call
E = dict(inval=uq.UQ_EINVAL, range=uq.UQ_ERANGE, align=uq.UQ_EALIGN, ws=uq.UQ_EWORKSPACE)


def quantize(x=A, type=0, rows=40, cols=70, ldx=72, stochastic=0, seed=1, codes=A, ldc=48, scales=A, lds=16, codes_t=A,
             ldct=32, scales_t=A, ldst=16):
    return L.uq_mx4_quantize(x, type, rows, cols, ldx, stochastic, seed, codes, ldc, scales, lds, codes_t, ldct, scales_t,
                             ldst, None)


def dequantize(codes=A, ldc=48, scales=A, lds=16, rows=40, cols=70, type=0, out=A, ldo=72):
    return L.uq_mx4_dequantize(codes, ldc, scales, lds, rows, cols, type, out, ldo, None)


def matmul(a=A, lda=48, sa=A, ldas=16, b=A, ldb=48, sb=A, ldbs=16, m=5, n=9, k=70, type=0, out=A, ldo=12, accumulate=0,
           ws=A, ws_bytes=1 << 30):
    return L.uq_mx4_matmul(a, lda, sa, ldas, b, ldb, sb, ldbs, m, n, k, type, out, ldo, accumulate, ws, ws_bytes, None)


def shared(g=A, d=100, rows=2, ldg=128, accumulate=0, scales=A):
    return L.uq_mx4_shared_scale(g, d, rows, ldg, accumulate, scales, None)


def qsum(g=A, d=100, rows=2, ldg=128, worker0=0, scales=A, seed=1, accumulate=0, sum_=A, M=2, out=A):
    return L.uq_mx4_quantize_sum(g, d, rows, ldg, worker0, scales, seed, accumulate, sum_, M, out, None)


def aggregate(g=A, d=100, M=2, ldg=128, seed=1, scales=A, sum_=A, out=A):
    return L.uq_mx4_aggregate(g, d, M, ldg, seed, scales, sum_, out, None)


def refused(status, want):
    assert status == E[want], uq.uq_last_error()
    assert uq.uq_last_error() != ""


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), "inval"), (dict(type=3), "range"), (dict(type=-1), "range"), (dict(rows=-1), "inval"),
    (dict(cols=-1), "inval"), (dict(rows=1 << 31), "range"), (dict(cols=1 << 31), "range"), (dict(ldx=68), "inval"),
    (dict(ldx=74), "align"), (dict(type=1, ldx=76), "align"), (dict(type=2, ldx=76), "align"), (dict(x=A + 8), "align"),
    (dict(stochastic=2), "inval"), (dict(stochastic=-1), "inval"), (dict(codes=None), "inval"),
    (dict(scales=None), "inval"), (dict(codes_t=None), "inval"), (dict(scales_t=None), "inval"),
    (dict(codes=None, scales=None, codes_t=None, scales_t=None), "inval"),
    (dict(ldc=32), "inval"), (dict(ldc=56), "align"), (dict(codes=A + 4), "align"), (dict(lds=0), "inval"),
    (dict(lds=8), "align"), (dict(scales=A + 1), "align"), (dict(ldct=16), "inval"), (dict(ldct=40), "align"),
    (dict(ldx=1 << 34), "range"), (dict(type=1, ldx=1 << 35), "range"), (dict(ldc=1 << 36), "range"),
    (dict(lds=1 << 36), "range"), (dict(ldct=1 << 36), "range"), (dict(ldst=1 << 36), "range"),
    (dict(codes_t=A + 8), "align"), (dict(ldst=1), "inval"), (dict(ldst=24), "align"), (dict(scales_t=A + 2), "align"),
])
def test_quantize_refuses(kw, want):
    refused(quantize(**kw), want)


@pytest.mark.parametrize("kw,want", [
    (dict(codes=None), "inval"), (dict(scales=None), "inval"), (dict(out=None), "inval"), (dict(type=7), "range"),
    (dict(rows=-2), "inval"), (dict(cols=1 << 31), "range"), (dict(ldc=32), "inval"), (dict(ldc=50), "align"),
    (dict(lds=2), "inval"), (dict(lds=20), "align"), (dict(ldo=64), "inval"), (dict(ldo=74), "align"),
    (dict(type=1, ldo=76), "align"), (dict(out=A + 4), "align"), (dict(codes=A + 2), "align"),
    (dict(ldo=1 << 34), "range"), (dict(ldc=1 << 36), "range"), (dict(lds=1 << 40), "range"),
    (dict(scales=A + 4), "align"),
])
def test_dequantize_refuses(kw, want):
    refused(dequantize(**kw), want)


@pytest.mark.parametrize("kw,want", [
    (dict(a=None), "inval"), (dict(sa=None), "inval"), (dict(b=None), "inval"), (dict(sb=None), "inval"),
    (dict(out=None), "inval"), (dict(ws=None), "inval"), (dict(ws=A + 8), "align"), (dict(ws_bytes=1), "ws"),
    (dict(m=-1), "inval"), (dict(n=-1), "inval"), (dict(k=-1), "inval"), (dict(m=1 << 31), "range"),
    (dict(n=1 << 31), "range"), (dict(k=1 << 31), "range"), (dict(type=3), "range"), (dict(accumulate=2), "inval"),
    (dict(lda=32), "inval"), (dict(lda=56), "align"), (dict(ldas=2), "inval"), (dict(ldas=12), "align"),
    (dict(ldb=32), "inval"), (dict(ldb=49), "align"), (dict(ldbs=0), "inval"), (dict(ldbs=17), "align"),
    (dict(lda=1 << 36), "range"), (dict(ldbs=1 << 36), "range"), (dict(ldo=1 << 34), "range"),
    (dict(ldo=8), "inval"), (dict(ldo=10), "align"), (dict(type=2, ldo=12), "align"), (dict(a=A + 8), "align"),
    (dict(sa=A + 4), "align"), (dict(b=A + 1), "align"), (dict(sb=A + 2), "align"), (dict(out=A + 4), "align"),
])
def test_matmul_refuses(kw, want):
    refused(matmul(**kw), want)


@pytest.mark.parametrize("kw,want", [
    (dict(g=None), "inval"), (dict(d=-1), "inval"), (dict(rows=0), "inval"), (dict(rows=70000), "range"),
    (dict(ldg=64), "inval"), (dict(ldg=130), "align"), (dict(g=A + 4), "align"), (dict(scales=None), "inval"),
    (dict(scales=A + 4), "align"), (dict(accumulate=3), "inval"),
])
def test_shared_scale_refuses(kw, want):
    refused(shared(**kw), want)


@pytest.mark.parametrize("kw,want", [
    (dict(g=None), "inval"), (dict(d=-1), "inval"), (dict(rows=0), "inval"), (dict(rows=70000), "range"),
    (dict(ldg=64), "inval"), (dict(ldg=130), "align"), (dict(g=A + 4), "align"), (dict(scales=None), "inval"),
    (dict(scales=A + 4), "align"), (dict(accumulate=-1), "inval"), (dict(worker0=-1), "range"),
    (dict(worker0=0x7FFFFFFF), "range"), (dict(sum_=None), "inval"), (dict(sum_=A + 4), "align"), (dict(M=0), "inval"),
    (dict(M=178956971), "range"), (dict(out=A + 8), "align"),
])
def test_quantize_sum_refuses(kw, want):
    refused(qsum(**kw), want)


@pytest.mark.parametrize("kw,want", [
    (dict(g=None), "inval"), (dict(d=-1), "inval"), (dict(M=0), "inval"), (dict(M=17), "range"), (dict(ldg=64), "inval"),
    (dict(ldg=130), "align"), (dict(g=A + 4), "align"), (dict(scales=None), "inval"), (dict(scales=A + 8), "align"),
    (dict(sum_=None), "inval"), (dict(sum_=A + 4), "align"), (dict(out=None), "inval"), (dict(out=A + 4), "align"),
])
def test_aggregate_refuses(kw, want):
    refused(aggregate(**kw), want)


def test_empty_calls_do_nothing():
    """No rows, no columns, no coordinates: accepted with no arrays at all and
    nothing launched (there is no GPU to launch on here)."""
    none = dict(codes=None, scales=None, codes_t=None, scales_t=None)
    assert quantize(x=None, rows=0, **none) == uq.UQ_OK and quantize(x=None, cols=0, **none) == uq.UQ_OK
    assert dequantize(codes=None, scales=None, out=None, rows=0) == uq.UQ_OK
    assert dequantize(codes=None, scales=None, out=None, cols=0) == uq.UQ_OK
    assert matmul(a=None, sa=None, out=None, m=0) == uq.UQ_OK
    assert matmul(b=None, sb=None, out=None, n=0) == uq.UQ_OK
    assert shared(d=0, g=None, scales=None) == uq.UQ_OK
    assert qsum(d=0, g=None, scales=None, sum_=None, out=None) == uq.UQ_OK
    assert aggregate(d=0, g=None, scales=None, sum_=None, out=None) == uq.UQ_OK


def test_workspace_is_never_zero_and_takes_any_size():
    for m, n, k in ((0, 0, 0), (1, 1, 1), (1, 8192, 8192), (4096, 4096, 1 << 20), (-5, 3, 1 << 40)):
        b = uq.uq_mx4_matmul_workspace_bytes(m, n, k)
        assert 0 < b < 1 << 32 and b % 256 == 0
