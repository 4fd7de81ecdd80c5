"""The 4-bit and layer-norm entry points as they are used together: a model that answers in 4 bits, replicas that train a norm,
deltas pushed in 4 bits; beside that random shapes on poisoned buffers, host threads and far offsets.

Tolerances are those of tests/test_gpu_fp4.py and tests/test_gpu_layer_norm.py, whose checks are used."""
import random
import threading

import numpy as np
import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.fp4_reference import Kept, encode, matrix
from tests.test_gpu_fp4 import DT, FORMATS, TYPES, check as check_product, check_codes, dequantize, product, quantize
from tests.test_gpu_layer_norm import backward, check_backward, check_forward, forward, params

pytestmark = pytest.mark.gpu


class Of:
    """What check() of a product wants to know of an operand that the library has quantised."""

    def __init__(self, x, fmt):
        self.q, self.s, self.t = quantize(x, fmt)
        codes, byte, t = encode(x, fmt)
        self.rows, self.cols, self.fmt = *x.shape, fmt
        self.values = torch.from_numpy(matrix(codes, byte, x.shape[1], fmt)).to(x.device)
        self.row = torch.ones(x.shape[0], dtype=torch.float64, device=x.device) if t is None else torch.from_numpy(t).to(x.device).double()


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 3, 16, 100, 700])
def test_a_model_that_answers_in_4_bits(cuda_device, M, dtype, fmt):
    """Norm, quantisation, hidden layer with bias and ReLU, twice, as one captured graph: each stage against its definition from
    the stage before, and the replays against each other."""
    g = torch.Generator(device=cuda_device).manual_seed(M)
    dims = [200, 512, 136]
    W = [Of(torch.randn(o, i, device=cuda_device, generator=g) / i ** 0.5, fmt) for i, o in zip(dims, dims[1:])]
    bias = [torch.randn(o, device=cuda_device, generator=g) for o in dims[1:]]
    par = [params(1, i, 3, cuda_device) for i in dims[:-1]]
    x = torch.randn(M, dims[0], device=cuda_device, generator=g).to(dtype)
    y = [torch.empty(M, i, device=cuda_device, dtype=dtype) for i in dims[:-1]]
    act = [x] + [torch.empty(M, o, device=cuda_device, dtype=dtype) for o in dims[1:]]
    room = [(torch.empty(M, (i + 31) // 32 * 16, dtype=torch.uint8, device=cuda_device),
             torch.empty(P.oscars_fp4_scale_bytes(M, i, fmt), dtype=torch.uint8, device=cuda_device),
             torch.empty(M, device=cuda_device) if fmt == P.NVFP4 else None) for i in dims[:-1]]

    def run():
        for l, (i, o) in enumerate(zip(dims, dims[1:])):
            q, s, t = room[l]
            P.oscars_layer_norm(act[l].data_ptr(), i, par[l][0].data_ptr(), par[l][1].data_ptr(), i, y[l].data_ptr(), i, DT[dtype], 1, M, i,
                                1e-5, stream=stream())
            P.oscars_quantize_fp4(y[l].data_ptr(), i, DT[dtype], M, i, fmt, q.data_ptr(), q.stride(0), s.data_ptr(),
                                  t.data_ptr() if t is not None else None, stream())
            P.oscars_gemm_fp4_nt(q.data_ptr(), q.stride(0), s.data_ptr(), W[l].q.data_ptr(), W[l].q.stride(0), W[l].s.data_ptr(), fmt,
                                 act[l + 1].data_ptr(), o, DT[dtype], M, o, i, t.data_ptr() if t is not None else None,
                                 W[l].t.data_ptr() if fmt == P.NVFP4 else None, bias[l].data_ptr(), True, stream())

    run()
    for l, i in enumerate(dims[:-1]):
        check_forward(act[l], *par[l], i, 1, M, y[l], None, None)
        check_product(act[l + 1], Of(y[l], fmt), W[l], bias[l], True)
    want = act[-1].clone()
    other = torch.randn(M, dims[0], device=cuda_device, generator=g).to(dtype)
    graph, s, first = torch.cuda.CUDAGraph(), torch.cuda.Stream(), x.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        run()
    x.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    check_product(act[-1], Of(y[-1], fmt), W[-1], bias[-1], True)
    x.copy_(first)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(act[-1], want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,batch,cols", [(16, 64, 512), (5, 33, 200), (3, 20, 1500)])
def test_replicas_train_a_norm_in_one_launch(cuda_device, workers, batch, cols, dtype):
    """W replicas' steps in one call are the steps of each alone: rows bit for bit, the parameters' sums as another
    order of the same sums, within the tolerance of both."""
    g = torch.Generator(device=cuda_device).manual_seed(workers)
    x = torch.randn(workers * batch, cols, device=cuda_device, generator=g).to(dtype)
    dy = torch.randn(workers * batch, cols, device=cuda_device, generator=g).to(dtype)
    gamma, beta = params(workers, cols, 5, cuda_device)
    for _ in range(3):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = forward(x, gamma, beta, cols, workers, batch, y)
        dg, db = (torch.empty(workers * cols, device=cuda_device) for _ in range(2))
        backward(dy, x, gamma, cols, mean, rstd, workers, batch, dx, dg, db, cols)
        check_forward(x, gamma, beta, cols, workers, batch, y, mean, rstd)
        check_backward(dy, x, gamma, cols, mean, rstd, workers, batch, dx, dg, db, cols)
        for w in range(workers):
            r = slice(w * batch, (w + 1) * batch)
            p = slice(w * cols, (w + 1) * cols)
            y1, dx1, dg1, db1 = torch.empty_like(y[r]), torch.empty_like(y[r]), torch.empty_like(dg[p]), torch.empty_like(db[p])
            m1, r1 = forward(x[r], gamma[p], beta[p], cols, 1, batch, y1)
            backward(dy[r], x[r], gamma[p], cols, m1, r1, 1, batch, dx1, dg1, db1, cols)
            assert torch.equal(y1, y[r]) and torch.equal(m1, mean[r]) and torch.equal(r1, rstd[r]) and torch.equal(dx1, dx[r])
            check_backward(dy[r], x[r], gamma[p], cols, m1, r1, 1, batch, None, dg1, db1, cols)
        gamma -= 0.01 * dg
        beta -= 0.01 * db


@pytest.mark.parametrize("fmt", FORMATS)
def test_deltas_pushed_in_4_bits(cuda_device, fmt):
    """Workers' deltas through 4 bits into the server's average: what arrives is what the codes stand for."""
    rows, cols, workers = 100, 333, 4
    g = torch.Generator(device=cuda_device).manual_seed(9)
    start = torch.randn(rows * cols, device=cuda_device, generator=g)
    got, exact = [], torch.zeros(rows, cols, dtype=torch.float64, device=cuda_device)
    for _ in range(workers):
        d = torch.randn(rows, cols, device=cuda_device, generator=g) * 0.01
        q, s, t = quantize(d, fmt)
        codes, byte, row = check_codes(d, fmt, q, s, t)
        got.append(dequantize(q, s, t, cols, fmt, torch.float32))
        v = torch.from_numpy(matrix(codes, byte, cols, fmt)).to(cuda_device)
        exact += (v if row is None else v * torch.from_numpy(row).to(cuda_device)[:, None].double()) / workers
    x = start.clone()
    P.oscars_merge(x.data_ptr(), [d.data_ptr() for d in got], [1.0 / workers] * workers, rows * cols, 1.0, stream())
    want = start.double() + exact.reshape(-1)
    # a delta is off by a rounding (its row's scale), the merge by one for each delta and the result's own
    tol = 2.0 ** -24 * (want.abs() + 8 * sum(d.abs().double() for d in got).reshape(-1) / workers) * 1.1
    assert ((x.double() - want).abs() <= tol).all()


def test_random_products_on_poisoned_buffers(cuda_device):
    """Shapes from every kernel and split, on buffers full of NaN, twice each: equal bits, and nothing around C touched."""
    rng = random.Random(3)
    for i in range(90):
        M, N = (int(round(2 ** rng.uniform(0, 10.3))) for _ in range(2))
        K = int(round(2 ** rng.uniform(0, 12.5 if M * N < 1 << 16 else 10)))
        fmt, dtype, relu = rng.choice(FORMATS), rng.choice(TYPES), rng.random() < 0.5
        A, B = Kept.random(M, K, fmt, cuda_device, i, pad=rng.choice([0, 16])), Kept.random(N, K, fmt, cuda_device, i + 1000)
        bias = torch.randn(N, device=cuda_device) if rng.random() < 0.5 else None
        ldc, shift = N + rng.choice([0, 0, 1, 8 - N % 8]), rng.choice([0, 0, 1])
        out = []
        for _ in range(2):
            buf = torch.full((shift + M * ldc + 40,), float("nan"), device=cuda_device, dtype=dtype)
            C = buf[shift:shift + M * ldc].view(M, ldc)[:, :N]
            product(A, B, dtype, bias, relu, C)
            rest = torch.ones_like(buf, dtype=torch.bool)
            rest[shift:shift + M * ldc].view(M, ldc)[:, :N] = False
            assert torch.isnan(buf[rest]).all(), (M, N, K)
            out.append(C.clone())
        assert torch.equal(out[0], out[1]), (M, N, K)
        check_product(out[0], A, B, bias, relu)


def test_host_threads(cuda_device):
    """Calls from threads at once, each on a stream of its own, are those of one after the other."""
    g = torch.Generator(device=cuda_device).manual_seed(6)
    jobs = []
    for i, size in enumerate([(1, 300, 200), (40, 300, 2100), (300, 520, 520), (600, 1024, 256)]):
        M, N, K = size
        fmt = FORMATS[i % 2]
        A, B = Kept.random(M, K, fmt, cuda_device, i), Kept.random(N, K, fmt, cuda_device, i + 7)
        out = torch.empty(M, N, device=cuda_device)
        jobs.append((lambda A=A, B=B, out=out: product(A, B, torch.float32, C=out), [out]))
    for groups, rows, cols in ((1, 900, 512), (4, 50, 1500)):
        x, dy = (torch.randn(groups * rows, cols, device=cuda_device, generator=g) for _ in range(2))
        gamma, beta = params(groups, cols, 1, cuda_device)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = (torch.empty(groups * rows, device=cuda_device) for _ in range(2))
        dg, db = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
        need = P.oscars_layer_norm_backward_workspace(groups, rows, cols)
        ws = torch.empty(need + 16, dtype=torch.uint8, device=cuda_device)

        def norm(x=x, dy=dy, gamma=gamma, beta=beta, y=y, dx=dx, mean=mean, rstd=rstd, dg=dg, db=db, ws=ws, need=need, n=(groups, rows, cols)):
            P.oscars_layer_norm(x.data_ptr(), n[2], gamma.data_ptr(), beta.data_ptr(), n[2], y.data_ptr(), n[2], P.F32, *n, 1e-5,
                                mean.data_ptr(), rstd.data_ptr(), stream())
            P.oscars_layer_norm_backward(dy.data_ptr(), n[2], x.data_ptr(), n[2], gamma.data_ptr(), n[2], mean.data_ptr(), rstd.data_ptr(),
                                         dx.data_ptr(), n[2], dg.data_ptr(), db.data_ptr(), n[2], P.F32, *n, ws.data_ptr(), need, stream())
        jobs.append((norm, [y, dx, mean, rstd, dg, db]))
    want = []
    for call, outs in jobs:
        call()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
        for o in outs:
            o.zero_()
    torch.cuda.synchronize()
    errors, go = [], threading.Barrier(len(jobs))

    def work(call):
        try:
            s = torch.cuda.Stream()
            go.wait()
            with torch.cuda.stream(s):
                for _ in range(60):
                    call()
            s.synchronize()
        except Exception as e:   # noqa: BLE001 (raised below)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c, _ in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors[0]
    for (_, outs), w in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))


def test_offsets_beyond_32_bits(cuda_device):
    """Rows 2^30 elements (or bytes) apart: their offsets pass 2^31 elements and 2^32 bytes."""
    far, K, N = 1 << 30, 100, 40
    g = torch.Generator(device=cuda_device).manual_seed(8)
    for fmt in FORMATS:
        x = torch.empty(5, far, dtype=torch.bfloat16, device=cuda_device)[:, :K]
        x.copy_(torch.randn(5, K, generator=g, device=cuda_device))
        q = torch.empty(5, far, dtype=torch.uint8, device=cuda_device)
        q[:, :64] = 0x5A
        s = torch.full((P.oscars_fp4_scale_bytes(5, K, fmt),), 0x5A, dtype=torch.uint8, device=cuda_device)
        t = torch.empty(5, device=cuda_device) if fmt == P.NVFP4 else None
        P.oscars_quantize_fp4(x.data_ptr(), far, P.BF16, 5, K, fmt, q.data_ptr(), far, s.data_ptr(), t.data_ptr() if t is not None else None,
                              stream())
        check_codes(x, fmt, q[:, :64], s, t)
        near = x.contiguous()
        x.zero_()
        P.oscars_dequantize_fp4(q.data_ptr(), far, s.data_ptr(), t.data_ptr() if t is not None else None, fmt, 5, K, x.data_ptr(), far, P.BF16,
                                stream())
        qn, sn, tn = quantize(near, fmt)
        assert torch.equal(x, dequantize(qn, sn, tn, K, fmt, torch.bfloat16))
        far_rows = Of(near, fmt)
        far_rows.q, far_rows.s, far_rows.t = q, s, t
        del x
        C = torch.empty(5, far, device=cuda_device)
        B = Kept.random(N, K, fmt, cuda_device, 1)
        check_product(product(far_rows, B, torch.float32, C=C[:, :N]), far_rows, B)
        del C
        for M in (1, 3, 20, 200):                         # channels far apart: every kernel
            A = Kept.random(M, K, fmt, cuda_device, 2)
            check_product(product(A, far_rows, torch.float32), A, far_rows)
        del q, far_rows
    for cols in (100, 777, 3001, 9000):
        rows = 3
        x, dy, y = (torch.empty(rows, far, dtype=torch.bfloat16, device=cuda_device)[:, :cols] for _ in range(3))
        x.copy_(torch.randn(rows, cols, generator=g, device=cuda_device))
        dy.copy_(torch.randn(rows, cols, generator=g, device=cuda_device))
        gamma, beta = params(1, cols, 1, cuda_device)
        mean, rstd = forward(x, gamma, beta, cols, 1, rows, y)
        check_forward(x, gamma, beta, cols, 1, rows, y, mean, rstd)
        dg, db = torch.empty(cols, device=cuda_device), torch.empty(cols, device=cuda_device)
        backward(dy, x, gamma, cols, mean, rstd, 1, rows, y, dg, db, cols)
        check_backward(dy, x, gamma, cols, mean, rstd, 1, rows, y, dg, db, cols)
        del x, dy, y


@pytest.mark.parametrize("rows,cols,at", [(1 << 20, 20800, [0, 127, 128, 700000, 823420, 823421, 825954, 825955, 900000, (1 << 20) - 1]),
                                          (70, (1 << 28) + 40, [0, 62, 63, 64, 69])])
def test_more_pieces_than_a_launch_takes(cuda_device, rows, cols, at):
    """1.3 x 2^30 and 1.1 x 2^30 pieces of 16 columns: two launches, the second from inside a scale tile on (MX: 2^30 / 1304 =
    823421 rows of eight pieces a tile, back: 2^30 / 1300 = 825955; of the wide matrix 63 rows)."""
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=cuda_device)
    g = torch.Generator(device=cuda_device).manual_seed(2)
    values = torch.randn(len(at), cols, generator=g, device=cuda_device).bfloat16()
    x[at] = values
    q = torch.empty(rows, (cols + 31) // 32 * 16, dtype=torch.uint8, device=cuda_device)
    s = torch.empty(P.oscars_fp4_scale_bytes(rows, cols, P.MXFP4), dtype=torch.uint8, device=cuda_device)
    P.oscars_quantize_fp4(x.data_ptr(), cols, P.BF16, rows, cols, P.MXFP4, q.data_ptr(), q.stride(0), s.data_ptr(), stream=stream())
    want = [quantize(v[None], P.MXFP4) for v in values]
    for r, (wq, _, _) in zip(at, want):
        assert torch.equal(q[r], wq[0])
    x.fill_(7.0)
    P.oscars_dequantize_fp4(q.data_ptr(), q.stride(0), s.data_ptr(), None, P.MXFP4, rows, cols, x.data_ptr(), cols, P.BF16, stream())
    for r, (wq, ws, _) in zip(at, want):
        assert torch.equal(x[r], dequantize(wq, ws, None, cols, P.MXFP4, torch.bfloat16)[0])
    for r in (1, 61, 65, rows // 2, rows - 2):
        assert (x[r] == 0).all()


def test_beside_the_8_bit_products_and_updates(cuda_device):
    """Streams with 4-bit products (pairs, clusters of eight) beside 8-bit products and orthogonalised updates, which all want an SM's
    tensor memory: each ends, with its own bits."""
    g = torch.Generator(device=cuda_device).manual_seed(1)
    jobs = []
    for i, (M, N, K) in enumerate([(100, 128, 5000), (700, 700, 700), (16, 600, 3000)]):
        A, B = Kept.random(M, K, FORMATS[i % 2], cuda_device, i), Kept.random(N, K, FORMATS[i % 2], cuda_device, i + 9)
        out = torch.empty(M, N, device=cuda_device)
        jobs.append((lambda A=A, B=B, out=out: product(A, B, torch.float32, C=out), out))
    for M, N, K in ((300, 500, 800), (40, 300, 2000)):
        A, B = (torch.randint(-128, 128, (r, K), dtype=torch.int8, generator=g, device=cuda_device) for r in (M, N))
        sa, sb, out = torch.rand(M, device=cuda_device), torch.rand(N, device=cuda_device), torch.empty(M, N, device=cuda_device)
        jobs.append((lambda A=A, B=B, sa=sa, sb=sb, out=out, n=(M, N, K): P.oscars_gemm_i8_nt(
            A.data_ptr(), n[2], sa.data_ptr(), B.data_ptr(), n[2], sb.data_ptr(), out.data_ptr(), n[1], P.F32, *n, stream=stream()), out))
    G, out = torch.randn(300, 400, generator=g, device=cuda_device), torch.empty(300, 400, device=cuda_device)
    ws = torch.empty(P.oscars_orthogonalize_workspace(1, 300, 400, P.F32), dtype=torch.uint8, device=cuda_device)
    jobs.append((lambda: P.oscars_orthogonalize(G.data_ptr(), 400, 0, out.data_ptr(), 400, 0, 1, 300, 400, P.F32, 5, ws.data_ptr(), ws.numel(),
                                                stream=stream()), out))
    want = []
    for call, o in jobs:
        call()
        torch.cuda.synchronize()
        want.append(o.clone())
        o.zero_()
    streams = [torch.cuda.Stream(priority=-(i % 2)) for i in range(len(jobs))]
    torch.cuda.synchronize()
    for _ in range(40):
        for s, (call, _) in zip(streams, jobs):
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for (_, o), w in zip(jobs, want):
        assert torch.equal(o, w)
