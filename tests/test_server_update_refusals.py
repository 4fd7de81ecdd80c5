"""What the orthogonalised update and the 8-bit product refuse, before any work on a
device (so it needs none): every call here is one that must not launch."""
import ctypes

import pytest

import paper_2102_08550_gb300 as P

NAN, INF = float("nan"), float("inf")
A = 1 << 20   # an aligned address that nothing reads


def refused(f, *a, **k):
    with pytest.raises(P.OscarsError) as e:
        f(*a, **k)
    assert e.value.status == P.OSCARS_EINVAL


def orth(g=A, ldg=8, bsg=64, o=A, ldo=8, bso=64, batch=1, rows=8, cols=8, dtype=0, steps=5, ws=A, n=1 << 40, **kw):
    P.oscars_orthogonalize(g, ldg, bsg, o, ldo, bso, batch, rows, cols, dtype, steps, ws, n, **kw)


@pytest.mark.parametrize("kw", [
    dict(g=0), dict(o=0), dict(ws=0), dict(ws=A + 128), dict(ws=A + 4), dict(n=0), dict(n=-1), dict(g=A + 2), dict(o=A + 1),
    dict(g=A + 1, dtype=1), dict(dtype=2), dict(dtype=-1), dict(ldg=7), dict(ldo=7), dict(ldg=-8), dict(bsg=-1), dict(bso=63, batch=2),
    dict(bso=0, batch=2), dict(bso=-64, batch=2), dict(batch=-1), dict(batch=65536), dict(rows=0), dict(cols=0), dict(rows=-3), dict(cols=65537, ldg=1 << 20, ldo=1 << 20),
    dict(rows=65537), dict(steps=0), dict(steps=65), dict(steps=-1), dict(eps=0.0), dict(eps=-1e-7), dict(eps=NAN), dict(eps=INF),
    dict(scale=NAN), dict(scale=INF), dict(coeff=(9, 0, 0)), dict(coeff=(0, -8.5, 0)), dict(coeff=(0, 0, NAN)), dict(coeff=(INF, 0, 0)),
    dict(coeff=(1, 2)), dict(coeff=(1, 2, 3, 4)), dict(coeff=(1, 4, 0.25)), dict(coeff=(1, 0.5, 1e-3)), dict(coeff=(1, 1e-5, 1e-8)),
])
def test_orthogonalize(oscars_lib, kw):
    refused(orth, **kw)


def test_the_workspace_is_measured(oscars_lib):
    for batch, rows, cols, dt in [(1, 1, 1, 0), (3, 100, 200, 1), (65535, 1, 1, 0), (1, 65536, 65536, 0)]:
        n = P.oscars_orthogonalize_workspace(batch, rows, cols, dt)
        assert n > 0
        refused(orth, batch=batch, rows=rows, cols=cols, ldg=cols, ldo=cols, bsg=rows * cols, bso=rows * cols, dtype=dt, n=n - 1)
    for bad in [(-1, 4, 4, 0), (1, 0, 4, 0), (1, 4, 65537, 0), (1, 4, 4, 7)]:
        refused(P.oscars_orthogonalize_workspace, *bad)
    refused(P.oscars_merge_orthogonal_workspace, 0, 4)
    assert oscars_lib.oscars_orthogonalize_workspace(1, 4, 4, 0, None) == P.OSCARS_EINVAL
    assert oscars_lib.oscars_merge_orthogonal_workspace(4, 4, None) == P.OSCARS_EINVAL


def test_an_empty_batch_is_no_work(oscars_lib):
    orth(batch=0, g=0, o=0, ws=0, n=0)
    refused(orth, batch=0, rows=0)


def merge(x=A, deltas=(A,), w=(1.0,), rows=8, cols=8, v=A, mu=0.9, nesterov=False, lr=0.1, steps=5, ws=A, n=1 << 40, **kw):
    P.oscars_merge_orthogonal(x, list(deltas), list(w), rows, cols, v, mu, nesterov, lr, steps, ws, n, **kw)


@pytest.mark.parametrize("kw", [
    dict(x=0), dict(x=A + 2), dict(v=A + 1), dict(deltas=(0,)), dict(deltas=(A + 3,)), dict(deltas=(), w=()), dict(deltas=[A] * 257, w=[0.1] * 257),
    dict(w=(1.0, 2.0)), dict(rows=0), dict(cols=-1), dict(rows=65537), dict(v=0, nesterov=True), dict(v=None, nesterov=True), dict(mu=NAN),
    dict(mu=INF), dict(lr=NAN), dict(lr=-INF), dict(steps=0), dict(ws=0), dict(ws=A + 64), dict(n=100), dict(eps=0.0), dict(coeff=(0, 0, 8.1)),
])
def test_merge_orthogonal(oscars_lib, kw):
    refused(merge, **kw)


def test_null_tables(oscars_lib):
    f = oscars_lib.oscars_merge_orthogonal
    one = (ctypes.c_float * 1)(1.0)
    tab = (ctypes.c_void_p * 1)(A)
    assert f(A, None, one, 1, 8, 8, A, 0.9, 0, 0.1, 5, None, 1e-7, A, 1 << 40, None) == P.OSCARS_EINVAL
    assert f(A, tab, None, 1, 8, 8, A, 0.9, 0, 0.1, 5, None, 1e-7, A, 1 << 40, None) == P.OSCARS_EINVAL


def quant(x=A, ldx=8, dtype=0, rows=4, cols=8, q=A, ldq=8, s=A):
    P.oscars_quantize_i8(x, ldx, dtype, rows, cols, q, ldq, s)


@pytest.mark.parametrize("kw", [dict(x=0), dict(q=0), dict(s=0), dict(x=A + 2), dict(x=A + 1, dtype=1), dict(s=A + 2), dict(ldx=7), dict(ldq=7),
                                dict(rows=-1), dict(cols=0), dict(dtype=2), dict(dtype=-1), dict(rows=(1 << 30) + 1),
                                dict(cols=(1 << 30) + 1, ldx=1 << 31, ldq=1 << 31)])
def test_quantize(oscars_lib, kw):
    refused(quant, **kw)


def product(a=A, lda=16, sa=A, b=A, ldb=16, sb=A, c=A, ldc=8, dtype=0, M=4, N=8, K=16, **kw):
    P.oscars_gemm_i8_nt(a, lda, sa, b, ldb, sb, c, ldc, dtype, M, N, K, **kw)


@pytest.mark.parametrize("kw", [
    dict(a=0), dict(b=0), dict(c=0), dict(sa=0), dict(sb=0), dict(a=A + 8), dict(b=A + 1), dict(sa=A + 1), dict(sb=A + 2), dict(bias_ptr=A + 2),
    dict(c=A + 2), dict(c=A + 1, dtype=1), dict(lda=15), dict(lda=24), dict(ldb=40), dict(lda=0), dict(K=17), dict(ldc=7), dict(M=-1), dict(N=0), dict(K=0),
    dict(K=131072, lda=131072, ldb=131072), dict(dtype=2), dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 1, ldc=1 << 31),
])
def test_gemm_i8(oscars_lib, kw):
    refused(product, **kw)


def test_no_tokens_is_no_work(oscars_lib):
    product(M=0, a=0, b=0, c=0, sa=0, sb=0)
    quant(rows=0, x=0, q=0, s=0)
