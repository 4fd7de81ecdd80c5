"""Orthogonalised updates over many shapes: random ones again and again on workspaces and results
full of anything (a store that is late or lost, or a buffer that is read before it is written,
changes a result only now and then), batches of many matrices, sides past 2048, and
coefficients at the limits that the call takes.  Tolerances: tests/test_gpu_orthogonal.py."""
import math
import random

import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.test_gpu_orthogonal import DT, check, orth, update

pytestmark = pytest.mark.gpu


def _shapes(seed, n):
    r = random.Random(seed)
    size = lambda lo, hi: int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))   # noqa: E731
    return [(size(1, 1400), size(1, 1400), r.choice([1, 1, 2, 3, 8]), r.choice([1, 2, 3, 5])) for _ in range(n // 2)] + \
           [(size(100, 1400), size(100, 1400), r.choice([1, 2, 4, 16, 24]), r.choice([1, 2, 3, 5])) for _ in range(n - n // 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seed", range(6))
def test_random_shapes_again_and_again(cuda_device, seed, dtype):
    for rows, cols, batch, steps in _shapes(seed, 10):
        G = torch.stack([update(rows, cols, 7 * seed + i, cuda_device) for i in range(batch)]).to(dtype)
        n = P.oscars_orthogonalize_workspace(batch, rows, cols, DT[dtype])
        ws, first = torch.empty(n, dtype=torch.uint8, device=cuda_device), None
        for rep in range(20):
            ws.fill_((37 * rep + 85) % 256)
            got = orth(G, steps, out=torch.full_like(G, float("nan")), ws=ws)
            if first is None:
                first = got
                for i in {0, batch - 1}:
                    check(got[i], G[i], steps)
            else:
                assert torch.equal(got, first), (rows, cols, batch, steps, rep)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,rows,cols", [(64, 10, 512), (433, 10, 512), (1024, 10, 512), (700, 33, 40), (65535, 2, 3), (200, 130, 70), (64, 64, 784),
                                             (48, 512, 300)])
def test_batches_of_many(cuda_device, batch, rows, cols, dtype):
    g = torch.Generator(device=cuda_device).manual_seed(batch)
    G = (torch.randn(batch, rows, cols, device=cuda_device, generator=g) * 1e-3).to(dtype)
    got = orth(G)
    for i in (0, 1, batch // 3, batch // 2, batch - 2, batch - 1):
        check(got[i], G[i], 5)
    assert torch.equal(orth(G), got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(2500, 2100), (2100, 5000), (4096, 2304), (4100, 4100)])
def test_both_sides_past_2048(cuda_device, rows, cols, dtype):
    G = update(rows, cols, rows + cols, cuda_device, rank=64).to(dtype)
    check(orth(G[None])[0], G, 5)


# b^2 = 32 |c| and b = 64 |c| at the limits; singular values stay below 2 over these steps
@pytest.mark.parametrize("steps,coeff", [(3, (0.5, 0.5, 1 / 128)), (2, (1.0, 0.25, 1 / 256)), (1, (4.8, -5.6, 1.0)), (1, (-2.0, 8.0, -2.0)),
                                         (3, (1.0, -0.5, 0.0079)), (8, (1.5, -0.5, 0.0)), (2, (0.0, 1.0, 0.0))])
@pytest.mark.parametrize("rows,cols", [(150, 260), (260, 150), (300, 300), (20, 40)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_coefficients_at_their_limits(cuda_device, rows, cols, steps, coeff, dtype):
    G = update(rows, cols, steps, cuda_device).to(dtype)
    check(orth(G[None], steps, coeff=coeff)[0], G, steps, coeff=coeff)
