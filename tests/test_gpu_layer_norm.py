"""Layer norm, forward and backward, against its definition in 64 bits.

Tolerances, u = 2^-24 (half a step of fp32).  A sum over a row of n values takes a value through at most D = 40 + n / 1024
additions (in a thread, over the lanes, over the warps), so it is off by D u times the sum of the magnitudes.
  mean: (D + 1) u mean|x|, called dm.
  var: each difference is rounded once and squared once, dm shifts it by dm^2: relative (D + 4) u + dm^2 / var; rstd half of
       that and 3 u of its own operations.
  y: |gamma| rstd (dm + u |x - mean|) + |gamma xh| (rstd's + 3 u) + u |y|, and half a step of its type.
  dx: a term of T = |h| + |mean h| + |xh mean(h xh)| + mean|h| + |xh| mean|h xh| takes at most D + 8 roundings; times rstd.
  dgamma, dbeta: a term takes at most 256 + rows / 64 additions (a thread's rows, a block's threads, the blocks) and 4 roundings."""
import pytest
import torch

import paper_2102_08550_gb300 as P

pytestmark = pytest.mark.gpu
DT = {torch.float32: P.F32, torch.bfloat16: P.BF16}
TYPES = [torch.float32, torch.bfloat16]
U = 2.0 ** -24
EPS = 1e-5
MORE = 1 + 2.0 ** -6   # second order


def stream():
    return torch.cuda.current_stream().cuda_stream


def ptr(t):
    return t.data_ptr() if t is not None else None


def half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def rows_at(values, pad, shift):
    """The rows `pad` elements further apart than their width, `shift` elements into a buffer of 7s."""
    r, c = values.shape
    buf = torch.full((shift + r * (c + pad) + 16,), 7.0, device=values.device, dtype=values.dtype)
    v = buf[shift:shift + r * (c + pad)].view(r, c + pad)[:, :c]
    v.copy_(values)
    return v, buf


def untouched(buf, r, c, pad, shift):
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[shift:shift + r * (c + pad)].view(r, c + pad)[:, :c] = False
    assert (buf[rest] == 7.0).all()


def params(groups, cols, seed, dev, stride=None):
    g = torch.Generator(device=dev).manual_seed(seed)
    stride = cols if stride is None else stride
    n = stride * (groups - 1) + cols
    return 1 + 0.3 * torch.randn(n, device=dev, generator=g), 0.2 * torch.randn(n, device=dev, generator=g)


def spread(p, groups, rows, cols, stride, none):
    """[groups * rows][cols] fp64 of parameters at a stride."""
    if p is None:
        return torch.full((1, 1), none, dtype=torch.float64, device="cuda")
    return torch.as_strided(p, (groups, cols), (stride, 1)).double().repeat_interleave(rows, 0)


def forward(x, gamma, beta, stride, groups, rows, y, eps=EPS, stats=True):
    cols = x.shape[1]
    mean, rstd = (torch.full((groups * rows,), 9.0, device=x.device) for _ in range(2)) if stats else (None, None)
    P.oscars_layer_norm(x.data_ptr(), x.stride(0), ptr(gamma), ptr(beta), stride, y.data_ptr(), y.stride(0), DT[x.dtype], groups, rows, cols, eps,
                        mean_ptr=ptr(mean), rstd_ptr=ptr(rstd), stream=stream())
    return mean, rstd


def check_forward(x, gamma, beta, stride, groups, rows, y, mean, rstd, eps=EPS):
    cols = x.shape[1]
    X, D = x.double(), 40 + cols / 1024
    m = X.mean(1, keepdim=True)
    d = X - m
    var = (d * d).mean(1, keepdim=True)
    r = (var + eps).rsqrt()
    g, b = spread(gamma, groups, rows, cols, stride, 1.0), spread(beta, groups, rows, cols, stride, 0.0)
    want = d * r * g + b
    dm = (D + 1) * U * X.abs().mean(1, keepdim=True)
    dr = 0.5 * ((D + 4) * U * var + dm * dm) / (var + eps) + 3 * U
    tol = g.abs() * r * (dm + U * d.abs()) + (g * d * r).abs() * (dr + 3 * U) + U * want.abs()
    tol = (tol * (1 + half_step(y.dtype)) + half_step(y.dtype) * want.abs()) * MORE + 1e-38
    bad = ~((y.double() - want).abs() <= tol)
    assert not bad.any(), (bad.sum().item(), bad.nonzero()[0].tolist())
    if mean is not None:
        assert ((mean.double() - m[:, 0]).abs() <= dm[:, 0] * MORE + 1e-38).all()
        assert ((rstd.double() - r[:, 0]).abs() <= (dr * r)[:, 0] * MORE).all()


def backward(dy, x, gamma, stride, mean, rstd, groups, rows, dx, dgamma, dbeta, dstride, ws=None):
    cols = x.shape[1]
    need = P.oscars_layer_norm_backward_workspace(groups, rows, cols)
    if ws is None:
        ws = torch.full((need // 4 + 4,), float("nan"), device=x.device)
    P.oscars_layer_norm_backward(dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), ptr(gamma), stride, mean.data_ptr(), rstd.data_ptr(),
                                 ptr(dx), dx.stride(0) if dx is not None else 0, ptr(dgamma), ptr(dbeta), dstride, DT[x.dtype], groups, rows,
                                 cols, ws.data_ptr(), need, stream=stream())


def check_backward(dy, x, gamma, stride, mean, rstd, groups, rows, dx, dgamma, dbeta, dstride):
    cols = x.shape[1]
    D = 40 + cols / 1024
    dY, g = dy.double(), spread(gamma, groups, rows, cols, stride, 1.0)
    r = rstd.double()[:, None]
    xh = (x.double() - mean.double()[:, None]) * r
    if dx is not None:
        h = dY * g
        sh, shx = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
        want = r * (h - sh - xh * shx)
        T = h.abs() + sh.abs() + (xh * shx).abs() + h.abs().mean(1, keepdim=True) + xh.abs() * (h * xh).abs().mean(1, keepdim=True)
        tol = r * T * (D + 8) * U
        tol = (tol * (1 + half_step(dx.dtype)) + half_step(dx.dtype) * want.abs()) * MORE + 1e-38
        bad = ~((dx.double() - want).abs() <= tol)
        assert not bad.any(), (bad.sum().item(), bad.nonzero()[0].tolist())
    depth = (256 + rows / 64 + 4) * U * MORE
    for got, terms in ((dgamma, dY * xh), (dbeta, dY)):
        if got is None:
            continue
        got = torch.as_strided(got, (groups, cols), (dstride, 1)).double()
        terms = terms.view(groups, rows, cols)
        bad = ~((got - terms.sum(1)).abs() <= depth * terms.abs().sum(1) + 1e-38)
        assert not bad.any(), (bad.sum().item(), bad.nonzero()[0].tolist())


def make(groups, rows, cols, dtype, dev, seed=0, pad=0, shift=0):
    g = torch.Generator(device=dev).manual_seed(seed * 1000003 + groups * 7919 + rows * 31 + cols)
    x = torch.randn(groups * rows, cols, device=dev, generator=g) * torch.exp(torch.randn(groups * rows, 1, device=dev, generator=g))
    x += torch.randn(groups * rows, 1, device=dev, generator=g)
    dy = torch.randn(groups * rows, cols, device=dev, generator=g)
    return rows_at(x.to(dtype), pad, shift)[0], rows_at(dy.to(dtype), pad, shift)[0]


# groups, rows, cols, pad, shift
SHAPES = [(1, 1, 1, 0, 0), (1, 1, 512, 0, 0), (1, 3, 2, 0, 0), (1, 5, 7, 3, 1), (2, 4, 8, 0, 0), (3, 5, 33, 7, 2), (16, 64, 512, 0, 0),
          (1, 1003, 777, 6, 0), (7, 33, 1000, 0, 0), (1, 130, 1024, 0, 0), (4, 70, 1025, 1, 3), (1, 9, 4096, 8, 0), (2, 100, 4097, 0, 0),
          (1, 40, 8192, 0, 0), (3, 7, 8191, 1, 0), (1, 12, 8200, 0, 0), (2, 3, 20001, 3, 5), (1, 2, 70000, 0, 0), (300, 2, 65, 0, 0),
          (2, 6, 3001, 2, 1), (1, 5, 5001, 3, 3), (3, 4, 8001, 0, 5), (1, 2500, 130, 0, 0), (32, 100, 96, 8, 8), (1, 700, 2048, 0, 0), (5, 257, 256, 0, 0), (65535, 1, 3, 0, 0), (2, 1500, 640, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,rows,cols,pad,shift", SHAPES)
def test_both_passes(cuda_device, groups, rows, cols, pad, shift, dtype):
    x, dy = make(groups, rows, cols, dtype, cuda_device, 1, pad, shift)
    gamma, beta = params(groups, cols, 2, cuda_device)
    y, ybuf = rows_at(torch.zeros(groups * rows, cols, device=cuda_device, dtype=dtype), pad, shift)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    check_forward(x, gamma, beta, cols, groups, rows, y, mean, rstd)
    untouched(ybuf, groups * rows, cols, pad, shift)
    dx, buf = rows_at(torch.zeros(groups * rows, cols, device=cuda_device, dtype=dtype), pad, shift)
    dgamma, dbeta = (torch.full((groups * cols + 4,), 7.0, device=cuda_device) for _ in range(2))
    backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    check_backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    untouched(buf, groups * rows, cols, pad, shift)
    assert (dgamma[groups * cols:] == 7).all() and (dbeta[groups * cols:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,rows,cols", [(1, 16384, 512), (1, 8192, 4096), (1, 3000, 8192), (16, 1000, 784), (1, 100000, 16)])
def test_large(cuda_device, groups, rows, cols, dtype):
    x, dy = make(groups, rows, cols, dtype, cuda_device, 3)
    gamma, beta = params(groups, cols, 4, cuda_device)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    check_forward(x, gamma, beta, cols, groups, rows, y, mean, rstd)
    dgamma, dbeta = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
    backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    check_backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,rows,cols", [(3, 20, 96), (2, 70, 1500), (2, 5, 9000)])
def test_parameters_shared_apart_or_absent(cuda_device, groups, rows, cols, dtype):
    x, dy = make(groups, rows, cols, dtype, cuda_device, 5)
    for stride in (0, cols + 3, cols + 8):
        gamma, beta = params(groups, cols, 6, cuda_device, stride)
        for g, b in ((gamma, beta), (None, beta), (gamma, None), (None, None)):
            y, dx = torch.empty_like(x), torch.empty_like(x)
            mean, rstd = forward(x, g, b, stride, groups, rows, y)
            check_forward(x, g, b, stride, groups, rows, y, mean, rstd)
            only = torch.empty_like(x)
            forward(x, g, b, stride, groups, rows, only, stats=False)
            assert torch.equal(only, y)
            dstride = cols + 5
            dgamma, dbeta = (torch.full((groups * dstride,), 7.0, device=cuda_device) for _ in range(2))
            backward(dy, x, g, stride, mean, rstd, groups, rows, dx, dgamma, dbeta, dstride)
            check_backward(dy, x, g, stride, mean, rstd, groups, rows, dx, dgamma, dbeta, dstride)
            assert (dgamma.view(groups, dstride)[:, cols:] == 7).all() and (dbeta.view(groups, dstride)[:, cols:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,rows,cols", [(1, 200, 512), (2, 70, 1500), (1, 9, 4096), (2, 5, 9000), (1, 3, 333)])
def test_in_place_and_wanted_parts(cuda_device, groups, rows, cols, dtype):
    """y over x, dx over dy or x, and each gradient alone: the bits of the full call."""
    x, dy = make(groups, rows, cols, dtype, cuda_device, 7)
    gamma, beta = params(groups, cols, 8, cuda_device)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    z = x.clone()
    forward(z, gamma, beta, cols, groups, rows, z)
    assert torch.equal(z, y)
    dgamma, dbeta = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
    backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    for over in (0, 1):
        a, b = dy.clone(), x.clone()
        g2, b2 = torch.empty_like(dgamma), torch.empty_like(dbeta)
        backward(a, b, gamma, cols, mean, rstd, groups, rows, (a, b)[over], g2, b2, cols)
        assert torch.equal((a, b)[over], dx) and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 0), (1, 0, 1), (0, 0, 0)):
        outs = [torch.full_like(t, 7.0) for t in (dx, dgamma, dbeta)]
        backward(dy, x, gamma, cols, mean, rstd, groups, rows, *(o if w else None for o, w in zip(outs, want)), cols)
        for o, w, full in zip(outs, want, (dx, dgamma, dbeta)):
            assert torch.equal(o, full) if w else (o == 7).all()


def test_no_rows(cuda_device):
    one = torch.ones(8, device=cuda_device)
    dgamma, dbeta = torch.full((8,), 7.0, device=cuda_device), torch.full((8,), 7.0, device=cuda_device)
    P.oscars_layer_norm_backward(0, 4, 0, 4, one.data_ptr(), 4, 0, 0, 0, 4, dgamma.data_ptr(), dbeta.data_ptr(), 4, P.F32, 2, 0, 4, 0, 0,
                                 stream=stream())
    assert (dgamma == 0).all() and (dbeta == 0).all()


@pytest.mark.parametrize("cols", [3, 100, 1024, 3000, 8192, 10000])
def test_values_over_fp32s_range(cuda_device, cols):
    """Rows of 2^120 and of 2^-60, of one value, with a far mean; a row with an infinity or NaN gives NaN and leaves the others."""
    g = torch.Generator(device=cuda_device).manual_seed(cols)
    x = torch.randn(9, cols, device=cuda_device, generator=g)
    clean = x.clone()
    x[1] *= 2.0 ** 120
    x[2] *= 2.0 ** -60
    x[3] = 0.0
    x[4] = 3.25
    x[5] = x[5] * 0.01 + 1000.0
    x[6, cols // 2] = float("inf")
    x[7, 0] = float("nan")
    x[1, 0] = 2.0 ** 126
    y, c = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = forward(x, None, None, 0, 1, 9, y)
    forward(clean, None, None, 0, 1, 9, c)
    good = [0, 1, 2, 3, 4, 5, 8]
    sub = x[good].contiguous()
    check_forward(sub, None, None, 0, 1, 7, y[good], mean[good], rstd[good])
    assert torch.isnan(y[6]).all() and torch.isnan(y[7]).all()
    assert torch.equal(y[0], c[0]) and torch.equal(y[8], c[8])
    x[8] = 2.0 ** 126   # the sum leaves fp32
    mean, rstd = forward(x, None, None, 0, 1, 9, y)
    assert mean[8] == 2.0 ** 126 and (y[8] == 0).all()


@pytest.mark.parametrize("eps", [1e-30, 1e-12, 1e-5, 1.0, 1e10])
def test_eps(cuda_device, eps):
    x, _ = make(1, 10, 300, torch.float32, cuda_device, 9)
    x[3] *= 1e-12
    x[4] = 0.5
    y = torch.empty_like(x)
    mean, rstd = forward(x, None, None, 0, 1, 10, y, eps)
    check_forward(x, None, None, 0, 1, 10, y, mean, rstd, float(torch.tensor(eps, dtype=torch.float32)))


@pytest.mark.parametrize("groups,rows,cols", [(1, 4, 40), (3, 5, 200)])
def test_gradients_against_differences(cuda_device, groups, rows, cols):
    """The derivative of sum(y w) along a direction, by central differences of the forward pass in 64 bits: off by h^2 / 6 of the
    third derivative, which h = 1e-4 leaves below 1e-6 of the gradient's own size, and by fp32's roundings, far below 1e-5 of it."""
    x, w = make(groups, rows, cols, torch.float32, cuda_device, 11)
    gamma, beta = params(groups, cols, 12, cuda_device)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    dgamma, dbeta = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
    backward(w, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)

    def loss(x, g, b):
        d = x - x.mean(1, keepdim=True)
        yy = d * ((d * d).mean(1, keepdim=True) + EPS).rsqrt() * g.repeat_interleave(rows, 0) + b.repeat_interleave(rows, 0)
        return (yy * w.double()).sum()

    at = [x.double(), gamma.view(groups, cols).double(), beta.view(groups, cols).double()]
    scale = x.double().std(1, keepdim=True)
    for i, grad in enumerate((dx, dgamma.view(groups, cols), dbeta.view(groups, cols))):
        for seed in range(4):
            v = torch.randn(at[i].shape, device=cuda_device, dtype=torch.float64, generator=torch.Generator(device=cuda_device).manual_seed(seed))
            if i == 0:
                v = v * scale
            h = 1e-4
            up, down = ([t + s * h * v if j == i else t for j, t in enumerate(at)] for s in (1, -1))
            numeric = (loss(*up) - loss(*down)) / (2 * h)
            size = (grad.double() * v).norm()
            assert ((grad.double() * v).sum() - numeric).abs() <= 1e-5 * size * v.numel() ** 0.5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,rows,cols", [(1, 1, 512), (16, 64, 512), (1, 2000, 1024), (1, 500, 4096), (2, 300, 9000)])
def test_repeats_on_streams_and_in_graphs(cuda_device, groups, rows, cols, dtype):
    cases = [make(groups, rows, cols, dtype, cuda_device, s) for s in (13, 14)]
    gamma, beta = params(groups, cols, 15, cuda_device)
    need = P.oscars_layer_norm_backward_workspace(groups, rows, cols)

    class Run:
        def __init__(self):
            self.y, self.dx = (torch.empty(groups * rows, cols, device=cuda_device, dtype=dtype) for _ in range(2))
            self.mean, self.rstd = (torch.empty(groups * rows, device=cuda_device) for _ in range(2))
            self.dg, self.db = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
            self.ws = torch.full((need // 4 + 4,), float("nan"), device=cuda_device)

        def __call__(self, x, dy):
            P.oscars_layer_norm(x.data_ptr(), cols, gamma.data_ptr(), beta.data_ptr(), cols, self.y.data_ptr(), cols, DT[dtype], groups, rows,
                                cols, EPS, self.mean.data_ptr(), self.rstd.data_ptr(), stream())
            P.oscars_layer_norm_backward(dy.data_ptr(), cols, x.data_ptr(), cols, gamma.data_ptr(), cols, self.mean.data_ptr(),
                                         self.rstd.data_ptr(), self.dx.data_ptr(), cols, self.dg.data_ptr(), self.db.data_ptr(), cols,
                                         DT[dtype], groups, rows, cols, self.ws.data_ptr(), need, stream())

        def all(self):
            return [self.y, self.mean, self.rstd, self.dx, self.dg, self.db]

    want = []
    for c in cases:
        run = Run()
        run(*c)
        want.append([t.clone() for t in run.all()])
    runs, streams = [Run(), Run()], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for r, s, c in zip(runs, streams, cases):
            with torch.cuda.stream(s):
                r(*c)
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        assert all(torch.equal(a, b) for a, b in zip(r.all(), w))
    graph, s, run = torch.cuda.CUDAGraph(), torch.cuda.Stream(), Run()
    inp = [t.clone() for t in cases[0]]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        run(*inp)
    for i in (1, 0):
        for a, b in zip(inp, cases[i]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(run.all(), want[i]))
