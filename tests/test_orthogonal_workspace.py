"""Workspaces of orthogonalised updates: what the call's own path touches and no more."""
import pytest

import paper_2102_08550_gb300 as P


@pytest.mark.parametrize("batch,rows,cols", [(1, 10, 512), (64, 10, 512), (7, 512, 10), (1, 1, 1), (1, 32, 1000), (16, 20, 30)])
def test_small_matrices_want_none_of_the_products_buffers(oscars_lib, batch, rows, cols):
    """One launch keeps them in shared memory: the status alone (64 matrices of 10 x 512 wanted 3 MB that nothing touched)."""
    assert P.oscars_orthogonalize_workspace(batch, rows, cols, P.F32) == 256


def test_a_server_step_on_one_wants_its_update(oscars_lib):
    """The merged update (4 bytes an element) and the sums of squares of its blocks."""
    n = P.oscars_merge_orthogonal_workspace(10, 512)
    assert 4 * 10 * 512 + 256 <= n <= 4 * 10 * 512 + 1024


def test_others_want_two_x_and_both_factors(oscars_lib):
    """In two halves of 16 bits each, rows on 128-byte lines; a bf16 result the rounding of A's diagonal too."""
    for dtype, more in ((P.F32, 0), (P.BF16, 3 * 512 * 4)):
        n = P.oscars_orthogonalize_workspace(3, 512, 784, dtype)
        want = 3 * (2 * 512 * 832 * 4 + 2 * 512 * 512 * 4) + more
        assert want < n <= want + 3 * 608 * 12 + 2048


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(10, 512), (512, 10), (1, 1), (33, 65), (64, 2000), (300, 200)])
def test_between_guards(cuda_device, rows, cols):
    import torch

    from tests.test_gpu_orthogonal import merge, orth, update
    for batch in (1, 5):
        G = torch.stack([update(rows, cols, i, cuda_device) for i in range(batch)])
        n = P.oscars_orthogonalize_workspace(batch, rows, cols, P.F32)
        buf = torch.full((n + 1024,), 77, dtype=torch.uint8, device=cuda_device)
        assert torch.equal(orth(G, ws=buf[512:512 + n]), orth(G))
        assert (buf[:512] == 77).all() and (buf[512 + n:] == 77).all()
    n = P.oscars_merge_orthogonal_workspace(rows, cols)
    buf = torch.full((n + 1024,), 77, dtype=torch.uint8, device=cuda_device)
    x, v = torch.zeros(rows, cols, device=cuda_device), torch.zeros(rows, cols, device=cuda_device)
    merge(x, [G[0]], [1.0], rows, cols, v, 0.9, False, 1.0, ws=buf[512:512 + n])
    assert (buf[:512] == 77).all() and (buf[512 + n:] == 77).all()
    # each within some 4e-6 of the definition; their norms are added up in another order
    assert (x - orth(G[:1])[0]).abs().max() <= 1e-5 * x.abs().max()
