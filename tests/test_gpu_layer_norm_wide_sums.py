"""Wide rows of the backward pass: a value goes through at most 40 + n / 1024 additions of a row's sums
(tests/test_gpu_layer_norm.py).

Column 0 has dy = 1, the others just under 2^-24, half a step of 1: added one after the other to 1 they are lost, and the
row's mean is off by 2^-24 / n for each of them.  Column 0's x is the mean, so that the other sum has no part in dx's bound."""
import pytest
import torch

from tests.test_gpu_layer_norm import backward, check_backward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [9000, 70000, 400000, 1000003])
def test_a_rows_sums_take_few_additions(cuda_device, cols, dtype):
    g = torch.Generator(device=cuda_device).manual_seed(cols)
    x = torch.randn(3, cols, device=cuda_device, generator=g).to(dtype)
    x[:, 0] = x.double().mean(1).to(dtype)
    dy = torch.full((3, cols), 1.9921875 * 2.0 ** -25, device=cuda_device, dtype=dtype)
    dy[:, 0] = 1.0
    y = torch.empty_like(x)
    mean, rstd = forward(x, None, None, 0, 1, 3, y)
    dx, dgamma, dbeta = torch.empty(3, cols, device=cuda_device, dtype=torch.float32).to(dtype), torch.empty(cols, device=cuda_device), torch.empty(cols, device=cuda_device)
    backward(dy, x, None, 0, mean, rstd, 1, 3, dx, dgamma, dbeta, cols)
    check_backward(dy, x, None, 0, mean, rstd, 1, 3, dx, dgamma, dbeta, cols)
