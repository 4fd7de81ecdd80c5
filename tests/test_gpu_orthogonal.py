"""Orthogonalised updates against Newton-Schulz steps in 64 bits.

Tolerance: four times the divergence of perturbed 64-bit runs on the same input
(tests/newton_schulz.py: each stored value moved within its rounding, each product
within its accumulation), plus half a step of the result's type: the factor covers
the roundings that the two seeds do not sample at their worst."""
import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.newton_schulz import envelope, newton_schulz

pytestmark = pytest.mark.gpu
DT = {torch.float32: P.F32, torch.bfloat16: P.BF16}


def update(rows, cols, seed, dev, rank=8, noise=0.3):
    g = torch.Generator(device=dev).manual_seed(seed)
    r = min(rank, rows, cols)
    u = torch.randn(rows, r, device=dev, generator=g) @ torch.randn(r, cols, device=dev, generator=g)
    return 1e-3 * (u / r ** 0.5 + noise * torch.randn(rows, cols, device=dev, generator=g))


def orth(G, steps=5, out=None, ws=None, stream=None, **kw):
    """G [batch, rows, cols] with any strides of rows and matrices."""
    b, r, c = G.shape
    O = torch.empty(b, r, c, dtype=G.dtype, device=G.device) if out is None else out
    if ws is None:
        ws = torch.empty(P.oscars_orthogonalize_workspace(b, r, c, DT[G.dtype]), dtype=torch.uint8, device=G.device)
    P.oscars_orthogonalize(G.data_ptr(), G.stride(1), G.stride(0), O.data_ptr(), O.stride(1), O.stride(0), b, r, c, DT[G.dtype],
                           steps, ws.data_ptr(), ws.numel(),
                           stream=torch.cuda.current_stream().cuda_stream if stream is None else stream, **kw)
    return O


def check(got, G, steps, **kw):
    ref, fro, big = envelope(G, steps, got.dtype, **kw)
    half = torch.finfo(got.dtype).eps / 2
    d = got.double() - ref
    assert torch.isfinite(got).all()
    assert d.norm() <= (4 * fro + half) * ref.norm(), (d.norm() / ref.norm(), fro)
    assert d.abs().max() <= (4 * big + half) * ref.abs().max(), (d.abs().max() / ref.abs().max(), big)


SIZES = [(1, 1), (1, 7), (7, 1), (1, 4096), (4096, 1), (2, 3), (8, 8), (10, 512), (512, 10), (16, 16), (17, 129), (31, 33),
         (64, 64), (65, 64), (127, 127), (128, 128), (128, 200), (129, 128), (130, 1000), (200, 64), (255, 300), (256, 256), (257, 511),
         (300, 257), (384, 1000), (512, 784), (784, 512), (777, 777)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_matches_64_bits(cuda_device, rows, cols, dtype):
    G = update(rows, cols, rows * 5000 + cols, cuda_device).to(dtype)
    check(orth(G[None])[0], G, 5)


@pytest.mark.parametrize("rows,cols", [(1024, 1024), (1000, 2050), (2050, 1000), (2048, 2048)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large(cuda_device, rows, cols, dtype):
    G = update(rows, cols, rows + cols, cuda_device, rank=64).to(dtype)
    check(orth(G[None])[0], G, 5)


@pytest.mark.parametrize("steps,coeff", [(1, None), (2, None), (8, None), (12, (1.5, -0.5, 0.0)), (6, (1.875, -1.25, 0.375)),
                                         (4, (2.0, -1.5, 0.5)), (3, (1.0, 0.0, 0.0)), (3, (1.5, 0.0, -0.5)), (2, (3.0, -4.0, 0.5))])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_and_coefficients(cuda_device, steps, coeff, dtype):
    G = update(150, 260, steps, cuda_device).to(dtype)
    kw = {} if coeff is None else {"coeff": coeff}
    check(orth(G[None], steps, **kw)[0], G, steps, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(33, 70), (70, 33), (200, 130), (12, 500)])
def test_batches_and_strides(cuda_device, rows, cols, dtype):
    """Rows and matrices apart from one another; what lies between them stays as it was."""
    b = 5
    buf = torch.full((b, rows + 3, cols + 5), 7.0, device=cuda_device, dtype=dtype)
    out = torch.full((b, rows + 2, cols + 3), 9.0, device=cuda_device, dtype=dtype)
    for i in range(b):
        buf[i, :rows, :cols] = (update(rows, cols, i, cuda_device) * 10.0 ** (i - 2)).to(dtype)
    before = buf.clone()
    G, O = buf[:, :rows, :cols], out[:, :rows, :cols]
    orth(G, out=O)
    for i in range(b):
        check(O[i], G[i], 5)
    assert torch.equal(buf, before)
    mask = torch.ones_like(out, dtype=torch.bool)
    mask[:, :rows, :cols] = False
    assert (out[mask] == 9.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place_and_one_matrix_for_all(cuda_device, dtype):
    G = update(100, 140, 3, cuda_device).to(dtype)
    alone = orth(G[None])[0]
    assert torch.equal(orth(G.clone()[None].contiguous()), alone[None])
    H = G.clone()[None]
    assert torch.equal(orth(H, out=H)[0], alone)
    many = orth(G[None].expand(4, 100, 140))
    for i in range(4):
        assert torch.equal(many[i], alone)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_any_alignment(cuda_device, shift):
    G = update(60, 48, 1, cuda_device)
    buf, out = torch.zeros(60 * 48 + 4, device=cuda_device), torch.zeros(60 * 48 + 4, device=cuda_device)
    buf[shift:shift + 2880] = G.reshape(-1)
    a, o = buf[shift:shift + 2880].view(1, 60, 48), out[shift:shift + 2880].view(1, 60, 48)
    assert torch.equal(orth(a, out=o), orth(G[None]))
    assert (out[:shift] == 0).all() and (out[shift + 2880:] == 0).all()


@pytest.mark.parametrize("rows,cols", [(40, 90), (300, 200)])
def test_the_norm_over_the_whole_range(cuda_device, rows, cols):
    """Updates far below and above where squares leave fp32: the result is that of the same update at size one."""
    G = update(rows, cols, 9, cuda_device) * 1e3
    one = orth(G[None], eps=1e-30)
    for power in (-90, -60, 60, 100):
        got = orth((G * 2.0 ** power)[None], eps=1e-30)
        tol = 1e-30 / (2.0 ** power * G.norm().item())   # what eps adds to the norm, where it counts
        assert (got - one).abs().max() <= max(1e-5, 500 * tol) * one.abs().max()


@pytest.mark.parametrize("rows,cols", [(1, 1), (20, 30), (300, 200), (140, 140)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_zeros_infinities_and_nan(cuda_device, rows, cols, dtype):
    Z = torch.zeros(2, rows, cols, device=cuda_device, dtype=dtype)
    assert (orth(Z) == 0).all()
    for bad in (float("inf"), float("-inf"), float("nan")):
        G = update(rows, cols, 2, cuda_device).to(dtype)[None].repeat(3, 1, 1)
        G[1, rows // 2, cols // 2] = bad
        got = orth(G)
        assert torch.isnan(got[1]).all()
        check(got[0], G[0], 5)   # its neighbours in the batch do not see it
        assert torch.equal(got[0], got[2])


def test_a_rank_of_one_and_empty_rows(cuda_device):
    """A single outer product becomes its direction; rows and columns of zeros stay zero."""
    g = torch.Generator(device=cuda_device).manual_seed(5)
    x, y = torch.randn(70, device=cuda_device, generator=g), torch.randn(90, device=cuda_device, generator=g)
    x[3], y[:5] = 0, 0
    G = 1e-3 * torch.outer(x, y)
    got = orth(G[None])[0]
    assert (got[3] == 0).all() and (got[:, :5] == 0).all()
    check(got, G, 5)


def test_empty_batch(cuda_device):
    P.oscars_orthogonalize(0, 4, 16, 0, 4, 16, 0, 4, 4, P.F32, 5, 0, 0)


@pytest.mark.parametrize("dtype,rows,cols,batch", [(torch.float32, 333, 120, 3), (torch.bfloat16, 512, 784, 2), (torch.float32, 20, 300, 2)])
def test_repeats_bit_for_bit_on_streams_and_in_graphs(cuda_device, dtype, rows, cols, batch):
    """The same bits on any stream, from a workspace full of anything, and replayed with other inputs."""
    G = torch.stack([update(rows, cols, i, cuda_device) for i in range(batch)]).to(dtype)
    H = torch.stack([update(rows, cols, 50 + i, cuda_device) for i in range(batch)]).to(dtype)
    want_g, want_h = orth(G), orth(H)
    n = P.oscars_orthogonalize_workspace(batch, rows, cols, DT[dtype])
    state = []
    torch.cuda.synchronize()
    for M, want in ((G, want_g), (H, want_h)):   # two at once, a workspace each
        s = torch.cuda.Stream()
        state.append((s, torch.full((n,), 255, dtype=torch.uint8, device=cuda_device), torch.empty_like(M), M, want))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, ws, out, M, _ in state:
            with torch.cuda.stream(s):
                orth(M, out=out, ws=ws)
    torch.cuda.synchronize()
    for _, _, out, _, want in state:
        assert torch.equal(out, want)
    s, ws, inp, out = torch.cuda.Stream(), torch.full((n,), 255, dtype=torch.uint8, device=cuda_device), G.clone(), torch.empty_like(G)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        orth(inp, out=out, ws=ws)
    for M, want in ((G, want_g), (H, want_h), (G, want_g)):
        inp.copy_(M)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_nothing_outside_the_workspace(cuda_device):
    """A workspace of exactly the bytes asked for, between guards."""
    for rows, cols, batch in [(10, 512, 1), (129, 65, 3), (65, 129, 2), (300, 300, 1)]:
        for dtype in (torch.float32, torch.bfloat16):
            G = torch.stack([update(rows, cols, i, cuda_device) for i in range(batch)]).to(dtype)
            n = P.oscars_orthogonalize_workspace(batch, rows, cols, DT[dtype])
            buf = torch.full((n + 1024,), 77, dtype=torch.uint8, device=cuda_device)
            assert buf.data_ptr() % 256 == 0
            orth(G, ws=buf[512:512 + n])
            assert (buf[:512] == 77).all() and (buf[512 + n:] == 77).all()


# ------------------------------------------------------------------ the server step
def merge(x, deltas, w, rows, cols, v, mu, nesterov, lr, steps=5, ws=None, **kw):
    if ws is None:
        ws = torch.empty(P.oscars_merge_orthogonal_workspace(rows, cols), dtype=torch.uint8, device=x.device)
    P.oscars_merge_orthogonal(x.data_ptr(), [d.data_ptr() for d in deltas], w, rows, cols,
                              v.data_ptr() if v is not None else None, mu, nesterov, lr, steps, ws.data_ptr(), ws.numel(),
                              stream=torch.cuda.current_stream().cuda_stream, **kw)


@pytest.mark.parametrize("rows,cols,W,shift,momentum,nesterov", [
    (1, 1, 1, 0, True, True), (10, 512, 16, 0, True, True), (512, 784, 3, 0, True, False), (33, 65, 1, 1, True, True),
    (129, 40, 8, 2, False, False), (257, 100, 9, 3, True, True), (100, 300, 17, 0, False, False), (64, 2000, 256, 0, True, False),
])
def test_server_step(cuda_device, rows, cols, W, shift, momentum, nesterov):
    n = rows * cols

    def shifted(t):
        buf = torch.full((n + 8,), 5.0, device=cuda_device)
        buf[shift:shift + n] = t.reshape(-1)
        return buf, buf[shift:shift + n]

    deltas = [shifted(update(rows, cols, 100 + k, cuda_device)) for k in range(W)]
    w = [(k + 1) / (W * (W + 1) / 2) for k in range(W)]
    xb, x = shifted(torch.rand(rows, cols, device=cuda_device) - 0.5)
    vb, v = shifted(update(rows, cols, 9, cuda_device))
    x0, v0 = x.clone(), v.clone()
    wf = torch.tensor(w, dtype=torch.float32).double()
    mu, lr = torch.tensor([0.95, 0.02], dtype=torch.float32).double().tolist()
    for step in range(2):   # two in a row: the momentum goes on
        x_old, v_old = x.double().clone(), v.double().clone()
        merge(x, [d for _, d in deltas], w, rows, cols, v if momentum else None, 0.95, nesterov, 0.02)
        d = sum(wk.item() * dk.double() for wk, (_, dk) in zip(wf, deltas))
        size = sum(abs(wk.item()) * dk.double().abs() for wk, (_, dk) in zip(wf, deltas))
        vr = mu * v_old + d if momentum else d
        u = (d + mu * vr if nesterov else vr).reshape(rows, cols)
        # W fused additions of the sum and one of the momentum, half a step each
        vtol = (W + 1) * 2.0 ** -24 * (size + mu * v_old.abs()) * (1 + 1e-5)
        if momentum:
            assert ((v.double() - vr).abs() <= vtol).all()
        else:
            assert torch.equal(v, v0)
        ref, fro, big = envelope(u.float(), 5, torch.float32)
        # the update's own rounding, (W + 2) half steps of its terms, goes through at most the steps' gain
        moved = newton_schulz(u + (W + 2) * 2.0 ** -24 * (size + 2 * v_old.abs()).reshape(rows, cols) *
                              torch.sign(torch.randn(rows, cols, dtype=torch.float64, device=cuda_device)), 5) - newton_schulz(u, 5)
        tol_fro = 4 * fro * ref.norm() + 4 * moved.norm()
        want = x_old + lr * newton_schulz(u, 5).reshape(-1)
        err = x.double() - want
        assert err.norm() <= lr * tol_fro + 2.0 ** -24 * want.norm() * 1.01, (err.norm(), lr * tol_fro)
    for buf in [xb, vb] + [b for b, _ in deltas]:
        assert (buf[:shift] == 5).all() and (buf[shift + n:] == 5).all()


def test_server_step_in_a_graph(cuda_device):
    """Replayed steps go on from the model and momentum that the last left."""
    rows, cols, W = 130, 70, 4
    deltas = [update(rows, cols, k, cuda_device) for k in range(W)]
    w = [0.25] * W

    def fresh():
        g = torch.Generator(device=cuda_device).manual_seed(3)
        return torch.randn(rows, cols, device=cuda_device, generator=g), torch.zeros(rows, cols, device=cuda_device)

    x, v = fresh()
    for _ in range(3):
        merge(x, deltas, w, rows, cols, v, 0.9, True, 0.1)
    y, u = fresh()
    ws = torch.empty(P.oscars_merge_orthogonal_workspace(rows, cols), dtype=torch.uint8, device=cuda_device)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        merge(y, deltas, w, rows, cols, u, 0.9, True, 0.1, ws=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x, y) and torch.equal(v, u)
