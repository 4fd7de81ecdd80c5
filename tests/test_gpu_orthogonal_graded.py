"""Orthogonalised updates whose rows or columns differ in size by many powers of
two: one row (a class, an embedding) with a far larger gradient than the others, and
rows that fall off evenly.  The norm is the whole matrix's, so the small rows' entries
are tiny; each step multiplies what lies in their directions by a, and after
enough of them it is as large as the rest of the result.

Tolerance, as in tests/test_gpu_orthogonal.py: four times the divergence of perturbed
64-bit runs on the same input, plus half a step of the result's type.  The
perturbations here know magnitudes: a value stored as fp16 halves is off by 2^-22 of itself
(two halves) or 2^-11 (one), and by half of fp16's smallest step (2^-25) over the power of
two that it is stored with: 2^12 for X and 2^8 for the factors, and 2^11 more for the
second half of an fp32 result's values.  A product is off by the accumulation's
2^-21 of the sum of its terms' magnitudes: the tensor core cuts up to 2^-23 of the running
sum at each of the four additions of a K-block's main product, and the average of what it
cuts is given back, so the errors have either sign."""
import pytest
import torch

from tests.newton_schulz import MUON, newton_schulz
from tests.test_gpu_orthogonal import merge, orth

pytestmark = pytest.mark.gpu
TWO, ONE, ACC = 2.0 ** -22, 2.0 ** -11, 2.0 ** -21
FLOOR_X = {torch.float32: 2.0 ** (-25 - 11 - 12), torch.bfloat16: 2.0 ** (-25 - 12)}
FLOOR_F = {torch.float32: 2.0 ** (-25 - 11 - 8), torch.bfloat16: 2.0 ** (-25 - 8)}


def perturbed(G, steps, dtype, gen, eps=1e-7):
    a, b, c = (torch.tensor(v, dtype=torch.float32).double().item() for v in MUON)

    def noise(x):
        return 2 * torch.rand(x.shape, generator=gen, dtype=x.dtype, device=x.device) - 1

    def store(x, rel, floor):
        return x + (rel * x.abs() + floor) * noise(x)

    def product(p, q):
        r = p @ q
        return r + ACC * (p.abs() @ q.abs()) * noise(r)

    factor = TWO if dtype == torch.float32 else ONE
    fx, ff = FLOOR_X[dtype], FLOOR_F[dtype]
    X = G.double()
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    X = X / (X.square().sum().sqrt() + torch.tensor(eps, dtype=torch.float32).double().item())
    X = store(X, TWO, fx)
    eye = torch.eye(X.shape[0], dtype=torch.float64, device=X.device)
    for k in range(steps):
        Y = X if dtype == torch.float32 else store(X, ONE, fx)
        A = store(product(Y, Y.T) + b / (2 * c) * eye, factor, ff)
        B = store((a - b * b / (4 * c)) * eye + c * product(A, A), factor, ff)
        X = store(product(B, Y if k + 1 == steps else X), TWO, fx)
    return X.T if tall else X


def tolerance(G, steps, dtype, eps=1e-7):
    ref = newton_schulz(G, steps, eps=eps)
    fro = big = 0.0
    for seed in (21, 22):
        d = perturbed(G, steps, dtype, torch.Generator(device=G.device).manual_seed(seed), eps) - ref
        fro, big = max(fro, d.norm().item()), max(big, d.abs().max().item())
    half = torch.finfo(dtype).eps / 2
    return ref, 4 * fro + half * ref.norm().item(), 4 * big + half * ref.abs().max().item()


def graded(kind, rows, cols, dev, seed=1):
    g = torch.Generator(device=dev).manual_seed(seed)
    G = torch.randn(rows, cols, device=dev, generator=g)
    name, size = kind
    if name == "row":
        G[rows // 3] *= size
    elif name == "column":
        G[:, cols // 3] *= size
    elif name == "rows":
        G *= torch.logspace(0, size, rows, device=dev)[:, None]
    else:
        G *= torch.logspace(0, size, cols, device=dev)[None]
    return 1e-3 * G


KINDS = [("row", 1e6), ("row", 1e5), ("row", 1e9), ("column", 1e6), ("rows", -8), ("columns", -8)]


@pytest.mark.parametrize("steps", [5, 8, 12])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(256, 512), (200, 260), (260, 200), (130, 1000), (60, 90)])
def test_rows_and_columns_of_different_sizes(cuda_device, rows, cols, kind, steps):
    for dtype in (torch.float32, torch.bfloat16):
        G = graded(kind, rows, cols, cuda_device).to(dtype)
        got = orth(G[None], steps)[0]
        ref, fro, big = tolerance(G, steps, dtype)
        d = got.double() - ref
        assert d.norm() <= fro, (dtype, (d.norm() / ref.norm()).item(), fro / ref.norm().item())
        assert d.abs().max() <= big, (dtype, (d.abs().max() / ref.abs().max()).item(), big / ref.abs().max().item())


@pytest.mark.parametrize("rows,cols", [(256, 512), (512, 200)])
def test_small_rows_come_up_in_a_server_step(cuda_device, rows, cols):
    """A step on a zero model is the orthogonalised merge itself."""
    G = graded(("row", 1e6) if rows < cols else ("column", 1e6), rows, cols, cuda_device)
    x = torch.zeros(rows, cols, device=cuda_device)
    merge(x, [G], [1.0], rows, cols, None, 0.0, False, 1.0, steps=12)
    ref, fro, big = tolerance(G, 12, torch.float32)
    d = x.double() - ref
    assert d.norm() <= fro and d.abs().max() <= big, (d.norm() / ref.norm(), fro / ref.norm())
