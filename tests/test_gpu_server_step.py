"""A server that applies orthogonalised updates and answers in 8 bits, as one program:
local steps of a context's workers push replicas, their deltas are merged into momentum,
orthogonalised and applied to each weight matrix (oscars_merge_orthogonal; the biases by
oscars_merge), the new weights are quantised, and a batch goes through the layers in
8 bits.  Every stage is checked against 64 bits from what the program itself held before
it, so that no stage's tolerance has to carry another's error."""
import threading

import pytest
import torch

import paper_2102_08550_gb300 as P
import synth
from tests.newton_schulz import envelope, newton_schulz
from tests.test_gpu_gemm_i8 import check as check_product, product, quantize

pytestmark = pytest.mark.gpu
MU, LR, STEPS = 0.9, 0.02, 5


def shapes(dims):
    return [(o, i) for i, o in zip(dims[:-1], dims[1:])]


def views(flat, dims):
    """[(W, b)] of a flat vector in canonical layout: whatever alignment the offsets give."""
    out, at = [], 0
    for o, i in shapes(dims):
        out.append((flat[at:at + o * i].view(o, i), flat[at + o * i:at + o * i + o]))
        at += o * i + o
    return out


def layer(x, Wq, sw, bias, relu, dtype):
    K = x.shape[1]
    ld = (K + 15) // 16 * 16
    A, sa = quantize(x, ld)
    return product(A, Wq, sa, sw, K, dtype, bias, relu), A, sa


@pytest.mark.parametrize("dims", [[130, 129, 10], [784, 512, 10], [100, 257, 65, 7]])
def test_rounds(cuda_device, dims):
    W, batch = 3, 32
    g = torch.Generator(device=cuda_device).manual_seed(sum(dims))
    P_total = sum(o * i + o for o, i in shapes(dims))
    x_g = (torch.rand(P_total, generator=g, device=cuda_device) - 0.5) * 0.2
    v = [torch.zeros(o, i, device=cuda_device) for o, i in shapes(dims)]
    ws = [torch.empty(P.oscars_merge_orthogonal_workspace(o, i), dtype=torch.uint8, device=cuda_device) for o, i in shapes(dims)]
    stream = torch.cuda.current_stream().cuda_stream
    weights = [0.5, 0.3, 0.2]
    x = torch.randn(70, dims[0], generator=g, device=cuda_device)
    for rnd in range(3):
        deltas = [1e-2 * torch.randn(P_total, generator=g, device=cuda_device) for _ in range(W)]
        old = x_g.clone()
        old_v = [t.clone() for t in v]
        dv = [views(d, dims) for d in deltas]
        for l, (o, i) in enumerate(shapes(dims)):
            Wl, bl = views(x_g, dims)[l]
            P.oscars_merge_orthogonal(Wl.data_ptr(), [dv[k][l][0].data_ptr() for k in range(W)], weights, o, i, v[l].data_ptr(), MU,
                                      True, LR, STEPS, ws[l].data_ptr(), ws[l].numel(), stream=stream)
            P.oscars_merge(bl.data_ptr(), [dv[k][l][1].data_ptr() for k in range(W)], weights, o, 1.0, stream)
        wf = torch.tensor(weights, dtype=torch.float32).double().tolist()
        mu, lr = torch.tensor([MU, LR], dtype=torch.float32).double().tolist()
        for l in range(len(dims) - 1):
            (Wl, bl), (Wo, bo) = views(x_g, dims)[l], views(old, dims)[l]
            d = sum(w * dv[k][l][0].double() for k, w in enumerate(wf))
            vr = mu * old_v[l].double() + d
            u = d + mu * vr
            assert (v[l].double() - vr).abs().max() <= 2.0 ** -22 * vr.abs().max() + 2.0 ** -22 * d.abs().max()
            _, fro, _ = envelope(u.float(), STEPS, torch.float32)
            O = newton_schulz(u, STEPS)
            err = Wl.double() - (Wo.double() + lr * O)
            # the update within four times its envelope (and as much again for u's own rounding), the sum within half a step
            assert err.norm() <= lr * 8 * fro * O.norm() + 2.0 ** -23 * Wl.double().norm()
            db = sum(w * dv[k][l][1].double() for k, w in enumerate(wf))
            assert (bl.double() - bo.double() - db).abs().max() <= 1e-6
        # the new model answers in 8 bits
        h = x
        for l, (Wl, bl) in enumerate(views(x_g, dims)):
            o, i = Wl.shape
            Wq, sw = quantize(Wl, (i + 15) // 16 * 16)
            last = l + 2 == len(dims)
            y, A, sa = layer(h, Wq, sw, bl.clone(), not last, torch.float32 if last else torch.bfloat16)
            check_product(y, A, Wq, sa, sw, i, bl, not last)
            h = y


def test_deltas_of_a_contexts_workers(cuda_device):
    """The replicas that local steps leave are the pushes: their deltas against the pulled model through the server step."""
    w = synth.TrainWorkload("server", 3, [256, 128, 10], 32, 0.05, 128, 4, 1, speeds=[1.0, 2.0, 1.5])
    shards = [synth.shard_t(w, k, cuda_device) for k in range(w.num_workers)]
    init = torch.from_numpy(synth.flatten_layers(synth.init_layers_np(w))).to(cuda_device)
    ctx = P.OscarsContext(num_workers=w.num_workers, dims=w.dims, batch=w.batch, lr=w.lr, speed=synth.speeds(w).tolist(), M=w.M,
                          shards=shards, init_params=init, stream=torch.cuda.current_stream().cuda_stream)
    x_g = torch.empty(ctx.P, device=cuda_device)
    ctx.pull(x_g)
    ctx.local_steps()
    deltas = []
    for k in range(w.num_workers):
        r = torch.empty(ctx.P, device=cuda_device)
        ctx.read_replica(k, r)
        deltas.append(r - x_g)
    ctx.push_merge()
    ctx.close()
    old = x_g.clone()
    for l, (Wl, _) in enumerate(views(x_g, w.dims)):
        o, i = Wl.shape
        ws = torch.empty(P.oscars_merge_orthogonal_workspace(o, i), dtype=torch.uint8, device=cuda_device)
        P.oscars_merge_orthogonal(Wl.data_ptr(), [views(d, w.dims)[l][0].data_ptr() for d in deltas], [1 / 3] * 3, o, i, None, 0.0, False,
                                  LR, STEPS, ws.data_ptr(), ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
        wf = torch.tensor(1 / 3, dtype=torch.float32).double().item()
        u = sum(wf * views(d, w.dims)[l][0].double() for d in deltas)
        _, fro, _ = envelope(u.float(), STEPS, torch.float32)
        O = newton_schulz(u, STEPS)
        lr = torch.tensor(LR, dtype=torch.float32).double().item()
        err = Wl.double() - (views(old, w.dims)[l][0].double() + lr * O)
        assert err.norm() <= lr * 8 * fro * O.norm() + 2.0 ** -23 * Wl.double().norm()


def test_a_step_and_its_answers_in_one_graph(cuda_device):
    """Copies and fills before and between the calls, all captured; replays go on from the last."""
    o, i, M = 200, 330, 40
    g = torch.Generator(device=cuda_device).manual_seed(1)

    def state():
        g.manual_seed(5)
        return {"x": torch.randn(o, i, generator=g, device=cuda_device) * 0.1, "v": torch.zeros(o, i, device=cuda_device),
                "d": torch.randn(o, i, generator=g, device=cuda_device) * 1e-2, "in": torch.empty(o, i, device=cuda_device),
                "t": torch.randn(M, i, generator=g, device=cuda_device).bfloat16(), "ld": 336,
                "Wq": torch.zeros(o, 336, dtype=torch.int8, device=cuda_device), "sw": torch.empty(o, device=cuda_device),
                "A": torch.zeros(M, 336, dtype=torch.int8, device=cuda_device), "sa": torch.empty(M, device=cuda_device),
                "y": torch.empty(M, o, device=cuda_device),
                "ws": torch.empty(P.oscars_merge_orthogonal_workspace(o, i), dtype=torch.uint8, device=cuda_device)}

    def step(s):
        st = torch.cuda.current_stream().cuda_stream
        s["in"].copy_(s["d"])          # a memory copy before the first call
        P.oscars_merge_orthogonal(s["x"].data_ptr(), [s["in"].data_ptr()], [1.0], o, i, s["v"].data_ptr(), MU, True, LR, STEPS,
                                  s["ws"].data_ptr(), s["ws"].numel(), stream=st)
        s["y"].zero_()                 # a fill between them
        P.oscars_quantize_i8(s["x"].data_ptr(), i, P.F32, o, i, s["Wq"].data_ptr(), 336, s["sw"].data_ptr(), stream=st)
        P.oscars_quantize_i8(s["t"].data_ptr(), i, P.BF16, M, i, s["A"].data_ptr(), 336, s["sa"].data_ptr(), stream=st)
        P.oscars_gemm_i8_nt(s["A"].data_ptr(), 336, s["sa"].data_ptr(), s["Wq"].data_ptr(), 336, s["sw"].data_ptr(),
                            s["y"].data_ptr(), o, P.F32, M, o, i, stream=st)
        s["d"].mul_(-0.7)              # a kernel of another library behind them

    a, b = state(), state()
    for _ in range(4):
        step(a)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        step(b)
    for _ in range(4):
        graph.replay()
    torch.cuda.synchronize()
    for k in ("x", "v", "Wq", "sw", "A", "sa", "y"):
        assert torch.equal(a[k], b[k]), k
    check_product(a["y"], a["A"], a["Wq"], a["sa"], a["sw"], i)


def test_threads_and_priorities(cuda_device):
    """Calls of several host threads on streams of both priorities give the bits that each gives alone."""
    jobs = []
    for n, (kind, size) in enumerate([("orth", (300, 500)), ("orth", (20, 700)), ("orth", (1024, 1024)), ("product", (16, 2000, 1000)),
                                      ("product", (500, 700, 900)), ("product", (1, 512, 784)), ("orth", (64, 64))]):
        g = torch.Generator(device=cuda_device).manual_seed(n)
        s = torch.cuda.Stream(priority=-1 if n % 2 else 0)
        if kind == "orth":
            G = torch.randn(*size, generator=g, device=cuda_device)
            O = torch.empty_like(G)
            ws = torch.empty(P.oscars_orthogonalize_workspace(1, *size, P.F32), dtype=torch.uint8, device=cuda_device)

            def call(G=G, O=O, ws=ws, s=s, size=size):
                P.oscars_orthogonalize(G.data_ptr(), size[1], 0, O.data_ptr(), size[1], 0, 1, *size, P.F32, 5, ws.data_ptr(),
                                       ws.numel(), stream=s.cuda_stream)
            out = O
        else:
            M, N, K = size
            ld = (K + 15) // 16 * 16
            A = torch.randint(-128, 128, (M, ld), dtype=torch.int8, generator=g, device=cuda_device)
            B = torch.randint(-128, 128, (N, ld), dtype=torch.int8, generator=g, device=cuda_device)
            sa, sb, C = torch.rand(M, device=cuda_device), torch.rand(N, device=cuda_device), torch.empty(M, N, device=cuda_device)

            def call(A=A, B=B, sa=sa, sb=sb, C=C, s=s, M=M, N=N, K=K, ld=ld):
                P.oscars_gemm_i8_nt(A.data_ptr(), ld, sa.data_ptr(), B.data_ptr(), ld, sb.data_ptr(), C.data_ptr(), N, P.F32, M, N, K,
                                    stream=s.cuda_stream)
            out = C
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        jobs.append((call, out, out.clone()))
    errors, go = [], threading.Barrier(len(jobs))

    def work(call):
        try:
            go.wait()
            for _ in range(150):
                call()
        except Exception as e:   # noqa: BLE001 (raised below)
            errors.append(e)
    for _, out, _ in jobs:
        out.zero_()
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c, _, _ in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors[0]
    for _, out, want in jobs:
        assert torch.equal(out, want)


def test_offsets_beyond_32_bits(cuda_device):
    """Rows 2^30 elements apart: their offsets pass 2^31 elements and 2^32 bytes."""
    far, K, N = 1 << 30, 100, 40
    g = torch.Generator(device=cuda_device).manual_seed(8)
    x = torch.empty(4, far, dtype=torch.bfloat16, device=cuda_device)[:, :K]
    x.copy_(torch.randn(4, K, generator=g, device=cuda_device))
    q = torch.empty(4, far, dtype=torch.int8, device=cuda_device)
    s = torch.empty(4, device=cuda_device)
    st = torch.cuda.current_stream().cuda_stream
    P.oscars_quantize_i8(x.data_ptr(), far, P.BF16, 4, K, q.data_ptr(), far, s.data_ptr(), stream=st)
    f = x.float()
    assert torch.equal(q[:, :K], torch.round(f / s[:, None]).to(torch.int8))
    near = q[:, :112].contiguous()
    B = torch.randint(-128, 128, (N, 112), dtype=torch.int8, generator=g, device=cuda_device)
    sb = torch.rand(N, generator=g, device=cuda_device)
    C = torch.empty(4, far, device=cuda_device)
    for M in (1, 2, 4):                                   # tokens far apart, the result's rows too
        P.oscars_gemm_i8_nt(q.data_ptr(), far, s.data_ptr(), B.data_ptr(), 112, sb.data_ptr(), C.data_ptr(), far, P.F32, M, N, K, stream=st)
        check_product(C[:M, :N], near[:M], B, s[:M], sb, K)
    A = torch.randint(-128, 128, (40, 112), dtype=torch.int8, generator=g, device=cuda_device)
    sa = torch.rand(40, generator=g, device=cuda_device)
    out = torch.empty(40, 4, device=cuda_device)
    for M in (1, 2, 20, 40):                              # channels far apart: every kernel
        P.oscars_gemm_i8_nt(A.data_ptr(), 112, sa.data_ptr(), q.data_ptr(), far, s.data_ptr(), out.data_ptr(), 4, P.F32, M, 4, K, stream=st)
        check_product(out[:M], A[:M], near, sa[:M], s, K)
    del C, q
    for rows, cols in ((4, 100), (4, 3000)):
        G = torch.empty(rows, far, device=cuda_device)[:, :cols]
        G.copy_(torch.randn(rows, cols, generator=g, device=cuda_device))
        O, want = torch.empty(rows, cols, device=cuda_device), torch.empty(rows, cols, device=cuda_device)
        ws = torch.empty(P.oscars_orthogonalize_workspace(1, rows, cols, P.F32), dtype=torch.uint8, device=cuda_device)
        P.oscars_orthogonalize(G.data_ptr(), far, 0, O.data_ptr(), cols, 0, 1, rows, cols, P.F32, 5, ws.data_ptr(), ws.numel(), stream=st)
        close = G.contiguous()
        P.oscars_orthogonalize(close.data_ptr(), cols, 0, want.data_ptr(), cols, 0, 1, rows, cols, P.F32, 5, ws.data_ptr(), ws.numel(),
                               stream=st)
        assert torch.equal(O, want)
        del G


def test_far_matrices_of_a_batch(cuda_device):
    """Matrices 2^31 elements apart, in and out (the tensor cores' path: 130 x 100)."""
    far, rows, cols = (1 << 31) + 64, 130, 100
    buf = torch.empty(far + rows * cols, device=cuda_device)
    g = torch.Generator(device=cuda_device).manual_seed(4)
    G = torch.randn(2, rows, cols, generator=g, device=cuda_device)
    for i in range(2):
        buf[i * far:i * far + rows * cols] = G[i].reshape(-1)
    want = torch.empty_like(G)
    ws = torch.empty(P.oscars_orthogonalize_workspace(2, rows, cols, P.F32), dtype=torch.uint8, device=cuda_device)
    st = torch.cuda.current_stream().cuda_stream
    P.oscars_orthogonalize(G.data_ptr(), cols, rows * cols, want.data_ptr(), cols, rows * cols, 2, rows, cols, P.F32, 5, ws.data_ptr(),
                           ws.numel(), stream=st)
    P.oscars_orthogonalize(buf.data_ptr(), cols, far, buf.data_ptr(), cols, far, 2, rows, cols, P.F32, 5, ws.data_ptr(), ws.numel(), stream=st)
    for i in range(2):
        assert torch.equal(buf[i * far:i * far + rows * cols].view(rows, cols), want[i])
