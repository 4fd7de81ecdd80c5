"""The parameters' gradients where few blocks have many rows: a term takes at most 256 + rows / 64 additions
(tests/test_gpu_layer_norm.py), however many groups there are and however wide a row is.

The first row of a group has dy = 1, the others just under 2^-24, half a step of 1: added one after the other to 1 they are all
lost, and the sum is off by 2^-24 for each of them."""
import pytest
import torch

from tests.test_gpu_layer_norm import backward, check_backward, forward, params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,rows,cols", [(77, 1000, 4104), (152, 700, 4200), (300, 600, 4104), (1, 3000, 40000), (20, 2000, 9000), (5, 12000, 600),
                                              (150, 9000, 100)])
def test_long_columns_are_added_up_in_short_runs(cuda_device, groups, rows, cols):
    g = torch.Generator(device=cuda_device).manual_seed(cols)
    x = torch.randn(groups * rows, cols, device=cuda_device, generator=g, dtype=torch.bfloat16)
    dy = torch.full((groups, rows, cols), 1.9921875 * 2.0 ** -25, device=cuda_device, dtype=torch.bfloat16)
    dy[:, 0] = 1.0
    dy = dy.view(groups * rows, cols)
    gamma, beta = params(groups, cols, 1, cuda_device)
    y = torch.empty_like(x)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    dgamma, dbeta = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
    dx = torch.empty_like(x)
    backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    check_backward(dy, x, gamma, cols, mean, rstd, groups, rows, None, dgamma, dbeta, cols)
    few = slice(0, rows)   # the first group's rows: the bits of a call of its own
    one, dg, db = torch.empty(rows, cols, device=cuda_device, dtype=torch.bfloat16), torch.empty(cols, device=cuda_device), torch.empty(cols, device=cuda_device)
    backward(dy[few], x[few], gamma, cols, mean[few], rstd[few], 1, rows, one, dg, db, cols)
    assert torch.equal(one, dx[few])
    # another order of the same terms
    check_backward(dy[few], x[few], gamma, cols, mean[few], rstd[few], 1, rows, None, dg, db, cols)
