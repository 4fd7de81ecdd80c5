"""bf16 orthogonalised updates are about as near to 64 bits as bf16 lets them be: their error is
held to 1.5 times that of the 64-bit result rounded to bf16, for up to eight steps.  (The
factors' roundings to 11 bits, 2^-12 of a value on average and relative to X, add up to about
bf16's own, 2^-8 over the square root of 12 in [1, 2), in five steps; of more, all but the last
three take two halves.)"""
import pytest
import torch

from tests.newton_schulz import newton_schulz
from tests.test_gpu_orthogonal import orth, update

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [1, 3, 5, 6, 8])
@pytest.mark.parametrize("rows,cols", [(10, 512), (64, 1000), (66, 3000), (80, 90), (100, 2000), (128, 128), (150, 700), (700, 150), (300, 300), (400, 4096),
                                       (512, 784), (784, 512), (1001, 333), (1024, 1024), (4096, 100)])
def test_as_near_as_bf16_results(cuda_device, rows, cols, steps):
    G = update(rows, cols, rows + cols, cuda_device, rank=64).bfloat16()
    ref = newton_schulz(G, steps)
    here, least = orth(G[None], steps)[0].double() - ref, ref.bfloat16().double() - ref
    assert here.norm() <= 1.5 * least.norm(), ((here.norm() / ref.norm()).item(), (least.norm() / ref.norm()).item())


@pytest.mark.parametrize("batch,rows,cols,steps", [(16, 512, 784, 5), (16, 512, 784, 8), (5, 200, 130, 6)])
def test_of_a_batch(cuda_device, batch, rows, cols, steps):
    G = torch.stack([update(rows, cols, i, cuda_device, rank=64) for i in range(batch)]).bfloat16()
    got = orth(G, steps)
    for i in range(batch):
        ref = newton_schulz(G[i], steps)
        assert (got[i].double() - ref).norm() <= 1.5 * (ref.bfloat16().double() - ref).norm()
