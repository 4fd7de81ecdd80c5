"""The status word of an orthogonalised update: zero after every call, whatever the workspace held."""
import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.test_gpu_orthogonal import DT, merge, orth, update

pytestmark = pytest.mark.gpu


def status(ws):
    return ws[:4].view(torch.int32).item()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,batch", [(10, 512, 1), (10, 512, 7), (300, 200, 1), (140, 140, 3), (512, 784, 16), (1024, 1024, 1)])
def test_zero_after_a_call(cuda_device, rows, cols, batch, dtype):
    G = torch.stack([update(rows, cols, i, cuda_device) for i in range(batch)]).to(dtype)
    n = P.oscars_orthogonalize_workspace(batch, rows, cols, DT[dtype])
    want = orth(G)
    for fill in (255, 1, 127):
        ws = torch.full((n,), fill, dtype=torch.uint8, device=cuda_device)
        assert torch.equal(orth(G, ws=ws), want) and status(ws) == 0
    ws, out = torch.full((n,), 255, dtype=torch.uint8, device=cuda_device), torch.empty_like(G)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        orth(G, out=out, ws=ws)
    for _ in range(2):
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and status(ws) == 0


@pytest.mark.parametrize("rows,cols", [(10, 512), (512, 784), (33, 65), (777, 130)])
def test_zero_after_a_server_step(cuda_device, rows, cols):
    d = [update(rows, cols, k, cuda_device) for k in range(3)]
    n = P.oscars_merge_orthogonal_workspace(rows, cols)
    got = []
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device=cuda_device)
        x, v = torch.zeros(rows, cols, device=cuda_device), torch.zeros(rows, cols, device=cuda_device)
        merge(x, d, [0.5, 0.3, 0.2], rows, cols, v, 0.9, True, 0.1, ws=ws)
        assert status(ws) == 0
        got.append((x, v))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
