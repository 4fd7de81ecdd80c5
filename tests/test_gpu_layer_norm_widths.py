"""Layer norm at the widths between powers of two: each number of warps a row, with rows on 16 bytes and off them, whole and cut
short, and results over their inputs where a row's copy begins in the row before.  Tolerances: tests/test_gpu_layer_norm.py."""
import pytest
import torch

from tests.test_gpu_layer_norm import TYPES, backward, check_backward, check_forward, forward, make, params, rows_at, untouched

pytestmark = pytest.mark.gpu
WIDTHS = [520, 768, 1032, 1536, 2056, 2560, 3000, 3080, 4096, 4104, 5000, 5120, 5128, 6000, 6144, 6152, 7000, 8184, 8192]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("groups,rows", [(1, 1), (2, 37), (1, 400)])
def test_rows_on_16_bytes(cuda_device, groups, rows, cols, dtype):
    x, dy = make(groups, rows, cols, dtype, cuda_device, 1, pad=8)
    gamma, beta = params(groups, cols, 2, cuda_device)
    y, ybuf = rows_at(torch.zeros(groups * rows, cols, device=cuda_device, dtype=dtype), 8, 0)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    check_forward(x, gamma, beta, cols, groups, rows, y, mean, rstd)
    untouched(ybuf, groups * rows, cols, 8, 0)
    dx, buf = rows_at(torch.zeros(groups * rows, cols, device=cuda_device, dtype=dtype), 8, 0)
    dgamma, dbeta = (torch.full((groups * cols + 4,), 7.0, device=cuda_device) for _ in range(2))
    backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    check_backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    untouched(buf, groups * rows, cols, 8, 0)
    assert (dgamma[groups * cols:] == 7).all() and (dbeta[groups * cols:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,rows,cols", [(1, 700, 3001), (2, 300, 1539), (1, 400, 4103), (3, 200, 5001), (1, 300, 8191), (2, 40, 9001), (1, 2000, 203)])
def test_results_over_rows_off_16_bytes(cuda_device, groups, rows, cols, dtype):
    """A block copies the last bytes of the row before its first one, which another block may be writing: they are not used."""
    x, dy = make(groups, rows, cols, dtype, cuda_device, 7)
    gamma, beta = params(groups, cols, 8, cuda_device)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = forward(x, gamma, beta, cols, groups, rows, y)
    check_forward(x, gamma, beta, cols, groups, rows, y, mean, rstd)
    dgamma, dbeta = (torch.empty(groups * cols, device=cuda_device) for _ in range(2))
    backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    check_backward(dy, x, gamma, cols, mean, rstd, groups, rows, dx, dgamma, dbeta, cols)
    for _ in range(5):
        z = x.clone()
        forward(z, gamma, beta, cols, groups, rows, z)
        assert torch.equal(z, y)
        for over in (0, 1):
            a, b = dy.clone(), x.clone()
            g2, b2 = torch.empty_like(dgamma), torch.empty_like(dbeta)
            backward(a, b, gamma, cols, mean, rstd, groups, rows, (a, b)[over], g2, b2, cols)
            assert torch.equal((a, b)[over], dx) and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)
