"""fp32 orthogonalised updates are about as near to 64 bits as the same steps in
fp32 products: their error is held to twice that of torch's on the same input.  (Values
have 22 bits for 24, but a sum is rounded every 64 terms instead of at each.)"""
import pytest
import torch

from tests.newton_schulz import MUON, newton_schulz
from tests.test_gpu_orthogonal import orth, update

pytestmark = pytest.mark.gpu


def in_fp32(G, steps):
    tall = G.shape[0] > G.shape[1]
    X = G.T if tall else G
    X = (X.double() / (X.double().norm() + 1e-7)).float()
    a, b, c = MUON
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if tall else X


@pytest.mark.parametrize("steps", [5, 8])
@pytest.mark.parametrize("rows,cols", [(10, 512), (60, 90), (80, 90), (100, 600), (333, 100), (200, 260), (130, 3000), (3000, 130), (512, 784),
                                       (1001, 333), (1024, 1024), (2048, 2048)])
def test_as_near_as_fp32_products(cuda_device, rows, cols, steps):
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        G = update(rows, cols, rows + cols, cuda_device, rank=64)
        ref = newton_schulz(G, steps)
        here, there = orth(G[None], steps)[0].double() - ref, in_fp32(G, steps).double() - ref
        assert here.norm() <= 2 * there.norm(), ((here.norm() / ref.norm()).item(), (there.norm() / ref.norm()).item())
    finally:
        torch.backends.cuda.matmul.allow_tf32 = tf32
