"""Orthogonalised updates whose norm, with eps, lies at either end of fp32's range.

Tolerances are those of tests/test_gpu_orthogonal.py: four times the divergence of
perturbed 64-bit runs on the same input, plus half a step of the result's type."""
import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.test_gpu_orthogonal import check, merge, orth, update

pytestmark = pytest.mark.gpu
SIZES = [(20, 30), (30, 20), (300, 200), (140, 140)]   # one launch, and products on the tensor cores


@pytest.mark.parametrize("eps", [3e38, 1e-7, 2.0 ** -126, 2.0 ** -127, 2.0 ** -128, 1e-39, 1e-42, 2.0 ** -149])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_zeros_give_zeros_with_every_eps(cuda_device, rows, cols, eps):
    for dtype in (torch.float32, torch.bfloat16):
        Z = torch.zeros(2, rows, cols, device=cuda_device, dtype=dtype)
        assert (orth(Z, eps=eps) == 0).all()


@pytest.mark.parametrize("rows,cols", SIZES)
def test_a_server_step_without_an_update_leaves_the_model(cuda_device, rows, cols):
    x = torch.randn(rows, cols, device=cuda_device)
    v, d, before = torch.zeros_like(x), torch.zeros_like(x), x.clone()
    for eps in (1e-7, 1e-39, 2.0 ** -149):
        merge(x, [d], [1.0], rows, cols, v, 0.9, True, 0.1, eps=eps)
        assert torch.equal(x, before) and (v == 0).all()


@pytest.mark.parametrize("power", [-149, -147, -140, -136, -130, -126, -120])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_updates_of_subnormal_numbers(cuda_device, rows, cols, power):
    """Whole multiples of 2^power: exact in fp32, with norms from 2^-144 on."""
    G = torch.round(update(rows, cols, 4, cuda_device).double() * 2e3).clamp(-100, 100) * 2.0 ** power
    assert torch.equal(G.float().double(), G) and (G != 0).any()
    G = G.float()
    for eps in (2.0 ** -149, 1e-40):
        check(orth(G[None], eps=eps)[0], G, 5, eps=eps)


@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** 124])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_updates_of_huge_numbers(cuda_device, rows, cols, dtype, size):
    """Norms up to 2^134, beyond fp32's range."""
    G = update(rows, cols, 5, cuda_device)
    G = (G / G.abs().max() * size * 8).to(dtype)
    assert torch.isfinite(G).all()
    check(orth(G[None])[0], G, 5)


@pytest.mark.parametrize("scale", [0.0, 1.0, -3.0, 1e38, 1e-30, 2.0 ** -110, 1e-35, -1e-36, 2.0 ** -130])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_every_scale(cuda_device, rows, cols, scale):
    """The result with a scale is that of one times it: four roundings of 2^-24, or 2^-150 each where it is subnormal."""
    G = update(rows, cols, 6, cuda_device)
    one, got = orth(G[None])[0].double(), orth(G[None], scale=scale)[0].double()
    want = one * torch.tensor(scale, dtype=torch.float32).double()
    assert torch.isfinite(got).all() and ((got - want).abs() <= 4 * (2.0 ** -24 * want.abs() + 2.0 ** -150)).all()
    H = G.bfloat16()
    one, got = orth(H[None])[0].double(), orth(H[None], scale=scale)[0].double()
    want = one * torch.tensor(scale, dtype=torch.float32).double()
    # both rounded to bf16, whose 8 bits are off by up to 2^-8 of a value (half a step of 2^-7 in [1, 2)), or 2^-134
    assert ((got - want).abs() <= 2.02 * 2.0 ** -8 * want.abs() + 2.0 ** -133).all()
