"""8-bit products whose scales lie at the ends of fp32's range: tokens of 1e37 have a scale
of 1e35, and their sums times it leave fp32, while the result does not where the channel's
scale is small; likewise below.

Tolerance, element by element: the sum is exact; its conversion, the two scales and a power
of two that moves a result into fp32's subnormal numbers are at most four roundings, each half a
step of fp32 (2^-24 of the value, or 2^-150), the bias one of the result, and the result's own
rounding half a step of its type (of bf16 2^-8, or 2^-134)."""
import pytest
import torch

from tests.test_gpu_gemm_i8 import codes, product

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TOKENS = [1.0, 2.0 ** 96, 2.0 ** 97, 1e30, 2.6e36, -3e37, 2.0 ** -126, 2.0 ** -127, 1e-40, 2.0 ** -149, 0.0, -1e-42, 3.4e38, 1e-30]
CHANNELS = [1.0, 1e-30, 3e-38, 1e-40, 1e-10, 1e10, 1e35, 3.4e38, 0.0, -1e-20, 2.0 ** -149, 1e20, 7e5]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 200, 100), (2, 130, 300), (1, 2000, 64), (2, 2000, 64), (8, 200, 100), (14, 300, 3000), (30, 260, 500),
                                   (33, 1024, 1024), (64, 260, 4096), (200, 300, 200), (300, 1000, 77), (1100, 2048, 130), (4000, 5000, 20)])
def test_only_the_result_decides_about_overflow(cuda_device, M, N, K, dtype):
    A, B = codes(M, K, 1, cuda_device), codes(N, K, 2, cuda_device)
    A[:, K // 2:K] = 0     # sums from a few to some 10^6
    A[M // 2:, 1:K] = 0
    B[3::7, :K] = 0        # sums of zero: zero with every finite scale
    exact = A[:, :K].double() @ B[:, :K].double().T
    for shift in range(0, len(TOKENS), max(1, M)):   # every token scale where there are few tokens
        sa = torch.tensor([TOKENS[(i + shift) % len(TOKENS)] for i in range(M)], device=cuda_device)
        sb = torch.tensor([CHANNELS[(i * 5 + i // 13) % len(CHANNELS)] for i in range(N)], device=cuda_device)
        for bias in (None, torch.randn(N, device=cuda_device)):
            prod = exact * sa.double()[:, None] * sb.double()
            want = prod if bias is None else prod + bias.double()
            got = product(A, B, sa, sb, K, dtype, bias, bias is not None)
            if bias is not None:
                want = want.clamp(min=0)
            top = torch.finfo(dtype).max
            tol = 4 * (U * prod.abs() + 2.0 ** -150) + (0 if bias is None else U * want.abs())
            if dtype == torch.bfloat16:
                tol = tol + torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -134
            tol = tol * (1 + 2.0 ** -6)
            assert not torch.isnan(got).any()
            over, under = want.abs() - tol > top * (1 + 2.0 ** -7), want.abs() + tol < top * (1 - 2.0 ** -7)
            assert torch.equal(got[over], torch.sign(want[over]).to(dtype) * float("inf"))
            bad = under & ((got.double() - want).abs() > tol)
            assert not bad.any(), (bad.sum().item(), bad.nonzero()[0].tolist(), sa[bad.nonzero()[0][0]].item(), sb[bad.nonzero()[0][1]].item())
