"""Layer norm's backward pass at the ends of fp32, at widths that fill a row's threads and at widths that leave some of their
columns behind the row's end: what stands behind it takes no part.  Tolerances: tests/test_gpu_layer_norm.py."""
import pytest
import torch

from tests.test_gpu_layer_norm import TYPES, backward, check_backward, forward, make, params, rows_at

pytestmark = pytest.mark.gpu
# one, some and all columns of the last turn; rows on one warp up to sixteen; past 8192 the passes of wide rows
COLS = [3, 100, 256, 512, 520, 777, 1024, 3000, 4096, 4104, 6000, 8192, 8200, 10000]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3)])
@pytest.mark.parametrize("cols", COLS)
def test_large_small_and_constant_rows(cuda_device, cols, pad, shift, dtype):
    """2^126 in all columns: x - mean is 0, and rstd 316 times a column of 0 behind the row's end, less the mean, leaves fp32."""
    g = torch.Generator(device=cuda_device).manual_seed(cols)
    x = torch.randn(9, cols, device=cuda_device, generator=g)
    x[1] *= 2.0 ** 100
    x[2] *= 2.0 ** -60
    x[3] = 0.0
    x[4] = 3.25
    x[5] = x[5] * 0.01 + 1000.0
    x[6] = 2.0 ** 126
    x[7] = -2.0 ** 126
    x = rows_at(x.to(dtype), pad, shift)[0]
    dy = rows_at(torch.randn(9, cols, device=cuda_device, generator=g).to(dtype), pad, shift)[0]
    gamma, beta = params(1, cols, 1, cuda_device)
    y, dx = (rows_at(torch.zeros(9, cols, device=cuda_device, dtype=dtype), pad, shift)[0] for _ in range(2))
    mean, rstd = forward(x, gamma, beta, cols, 1, 9, y)
    assert mean[6] == 2.0 ** 126 and mean[7] == -2.0 ** 126
    dgamma, dbeta = torch.empty(cols, device=cuda_device), torch.empty(cols, device=cuda_device)
    for g in (gamma, None):
        backward(dy, x, g, cols, mean, rstd, 1, 9, dx, dgamma, dbeta, cols)
        check_backward(dy, x, g, cols, mean, rstd, 1, 9, dx, dgamma, dbeta, cols)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("eps", [1e-38, 1e-30, 1e-12, 1.0, 1e10])
def test_eps(cuda_device, eps, cols):
    """Constant rows under a small eps: rstd is 1e19 at most, and 2^66 times that leaves fp32."""
    x, dy = make(1, 10, cols, torch.float32, cuda_device, 9)
    x[3] *= 1e-12
    x[4] = 0.5
    x[5] = 2.0 ** 66
    x[6] = -2.0 ** 100
    y, dx = torch.empty_like(x), torch.empty_like(x)
    gamma, beta = params(1, cols, 1, cuda_device)
    mean, rstd = forward(x, gamma, beta, cols, 1, 10, y, eps)
    dgamma, dbeta = torch.empty(cols, device=cuda_device), torch.empty(cols, device=cuda_device)
    backward(dy, x, gamma, cols, mean, rstd, 1, 10, dx, dgamma, dbeta, cols)
    check_backward(dy, x, gamma, cols, mean, rstd, 1, 10, dx, dgamma, dbeta, cols)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_rows_without_a_number_leave_the_others(cuda_device, cols, dtype):
    x, dy = make(1, 7, cols, dtype, cuda_device, 11)
    gamma, beta = params(1, cols, 1, cuda_device)
    bad = x.clone()
    bad[2, cols // 2] = float("nan")
    bad[5, 0] = float("inf")
    outs = []
    for v in (x, bad):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = forward(v, gamma, beta, cols, 1, 7, y)
        dgamma, dbeta = torch.empty(cols, device=cuda_device), torch.empty(cols, device=cuda_device)
        backward(dy, v, gamma, cols, mean, rstd, 1, 7, dx, dgamma, dbeta, cols)
        outs.append((y, dx, dbeta))
    keep = [0, 1, 3, 4, 6]
    for a, b in zip(*outs):
        if a.dim() == 2:
            assert torch.equal(a[keep], b[keep]) and torch.isnan(b[[2, 5]]).all()
        else:
            assert torch.equal(a, b)   # dbeta knows nothing of x
