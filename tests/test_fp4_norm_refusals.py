"""What the 4-bit and layer-norm entry points refuse, before any device work (no GPU needed)."""
import pytest

import paper_2102_08550_gb300 as P

BIG = (1 << 30) + 1


def refused(f):
    with pytest.raises(P.OscarsError) as e:
        f()
    assert e.value.status == P.OSCARS_EINVAL


def quantize(x=4096, ldx=64, dtype=P.F32, rows=4, cols=64, fmt=P.NVFP4, q=4096, ldq=32, s=4096, t=4096):
    P.oscars_quantize_fp4(x, ldx, dtype, rows, cols, fmt, q, ldq, s, t)


@pytest.mark.parametrize("kw", [dict(x=0), dict(x=4098), dict(x=4097, dtype=P.BF16), dict(ldx=63), dict(dtype=2), dict(rows=-1), dict(rows=BIG),
                                dict(cols=0), dict(cols=BIG, ldx=BIG, ldq=1 << 30), dict(fmt=2), dict(fmt=-1), dict(q=0), dict(q=4104),
                                dict(ldq=16), dict(ldq=40), dict(s=0), dict(s=4100), dict(t=None), dict(t=4098), dict(fmt=P.MXFP4),
                                dict(cols=65, ldx=65)])
def test_quantize(oscars_lib, kw):
    refused(lambda: quantize(**kw))


def dequantize(q=4096, ldq=32, s=4096, t=4096, fmt=P.NVFP4, rows=4, cols=64, x=4096, ldx=64, dtype=P.F32):
    P.oscars_dequantize_fp4(q, ldq, s, t, fmt, rows, cols, x, ldx, dtype)


@pytest.mark.parametrize("kw", [dict(q=0), dict(q=4100), dict(ldq=31), dict(ldq=16), dict(s=0), dict(s=4104), dict(t=4097), dict(fmt=7),
                                dict(rows=-2), dict(rows=BIG), dict(cols=0), dict(cols=BIG), dict(x=0), dict(x=4097, dtype=P.BF16),
                                dict(ldx=10), dict(dtype=-1)])
def test_dequantize(oscars_lib, kw):
    refused(lambda: dequantize(**kw))


def product(a=4096, lda=32, sa=4096, b=4096, ldb=32, sb=4096, fmt=P.MXFP4, c=4096, ldc=8, dtype=P.F32, M=4, N=8, K=64, **kw):
    P.oscars_gemm_fp4_nt(a, lda, sa, b, ldb, sb, fmt, c, ldc, dtype, M, N, K, **kw)


@pytest.mark.parametrize("kw", [dict(a=0), dict(a=4097), dict(lda=24), dict(lda=16), dict(sa=0), dict(sa=4100), dict(b=0), dict(b=4104),
                                dict(ldb=0), dict(ldb=33), dict(sb=0), dict(sb=4097), dict(fmt=3), dict(c=0), dict(c=4098),
                                dict(c=4097, dtype=P.BF16), dict(ldc=7), dict(dtype=5), dict(M=-1), dict(M=BIG), dict(N=0), dict(N=BIG, ldc=BIG),
                                dict(K=0), dict(K=BIG), dict(K=65), dict(lda=1 << 40), dict(ldb=1 << 40), dict(row_scale_a_ptr=4097), dict(row_scale_b_ptr=4098), dict(bias_ptr=4099)])
def test_product(oscars_lib, kw):
    refused(lambda: product(**kw))


@pytest.mark.parametrize("args", [(-1, 8, 0), (8, 0, 0), (BIG, 8, 0), (8, BIG, 1), (8, 8, 2)])
def test_scale_bytes(oscars_lib, args):
    refused(lambda: P.oscars_fp4_scale_bytes(*args))


def test_scale_bytes_are_whole_tiles(oscars_lib):
    for rows, cols, fmt, tiles in ((1, 1, P.MXFP4, 1), (128, 128, P.MXFP4, 1), (129, 128, P.MXFP4, 2), (128, 129, P.MXFP4, 2),
                                   (128, 128, P.NVFP4, 2), (1000, 65, P.NVFP4, 16), (1 << 30, 1 << 30, P.NVFP4, (1 << 23) * (1 << 24))):
        assert P.oscars_fp4_scale_bytes(rows, cols, fmt) == tiles * 512


def norm(x=4096, ldx=64, gamma=4096, beta=4096, stride=64, y=8192, ldy=64, dtype=P.F32, groups=2, rows=3, cols=64, eps=1e-5, **kw):
    P.oscars_layer_norm(x, ldx, gamma, beta, stride, y, ldy, dtype, groups, rows, cols, eps, **kw)


NAN, INF = float("nan"), float("inf")
SIZES = [dict(groups=-1), dict(groups=65536), dict(rows=-1), dict(rows=BIG), dict(groups=2, rows=(1 << 29) + 1), dict(cols=0), dict(cols=BIG), dict(dtype=2)]


@pytest.mark.parametrize("kw", SIZES + [dict(x=0), dict(x=4098), dict(x=4097, dtype=P.BF16), dict(ldx=63), dict(gamma=4097), dict(beta=4098),
                                        dict(stride=-1), dict(y=0), dict(y=8193), dict(ldy=63), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN),
                                        dict(eps=INF), dict(mean_ptr=4097), dict(rstd_ptr=4098), dict(y=4096, ldx=64, ldy=80)])
def test_layer_norm(oscars_lib, kw):
    refused(lambda: norm(**kw))


def backward(dy=4096, lddy=64, x=8192, ldx=64, gamma=4096, stride=64, mean=4096, rstd=4096, dx=16384, lddx=64, dgamma=4096, dbeta=4096,
             dstride=64, dtype=P.F32, groups=2, rows=3, cols=64, ws=4096, ws_bytes=1 << 40):
    P.oscars_layer_norm_backward(dy, lddy, x, ldx, gamma, stride, mean, rstd, dx, lddx, dgamma, dbeta, dstride, dtype, groups, rows, cols, ws,
                                 ws_bytes)


@pytest.mark.parametrize("kw", SIZES + [dict(dy=0), dict(dy=4098), dict(x=0), dict(x=8193, dtype=P.BF16), dict(lddy=63), dict(ldx=1), dict(lddx=63),
                                        dict(gamma=4097), dict(stride=-4), dict(mean=0), dict(rstd=0), dict(mean=4098), dict(rstd=4097),
                                        dict(dx=16385), dict(dx=4096, lddx=72), dict(dx=8192, lddx=72), dict(dgamma=4098), dict(dbeta=4097),
                                        dict(dstride=63), dict(ws=4104), dict(rows=10000, ws_bytes=64), dict(rows=10000, ws=0)])
def test_layer_norm_backward(oscars_lib, kw):
    refused(lambda: backward(**kw))


@pytest.mark.parametrize("args", [(-1, 8, 8), (65536, 8, 8), (1, -1, 8), (1, BIG, 8), (1, 8, 0), (1, 8, BIG), (4, 1 << 29, 8)])
def test_layer_norm_backward_workspace(oscars_lib, args):
    refused(lambda: P.oscars_layer_norm_backward_workspace(*args))


def test_nothing_to_do(oscars_lib):
    norm(x=0, y=0, groups=0)
    norm(x=0, y=0, rows=0)
    backward(dy=0, x=0, mean=0, rstd=0, groups=0)
    assert P.oscars_layer_norm_backward_workspace(0, 5, 5) >= 0
