"""8-bit products against exact integer sums, rows' codes against fp32 division.

Tolerance of a product, element by element: the sum is exact; its conversion and
the two scales are three roundings of the product, the bias one of the result, each
half a step of fp32 (2^-24), and the result's own rounding half a step of its type."""
import pytest
import torch

import paper_2102_08550_gb300 as P

pytestmark = pytest.mark.gpu
DT = {torch.float32: P.F32, torch.bfloat16: P.BF16}
U = 2.0 ** -24


def codes(rows, K, seed, dev, pad=0, lo=-128, hi=128):
    """int8 rows, K columns of them used; the bytes behind are anything."""
    ld = (K + 15) // 16 * 16 + pad
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.randint(lo, hi, (rows, ld), device=dev, generator=g, dtype=torch.int8)


def product(A, B, sa, sb, K, dtype, bias=None, relu=False, C=None):
    M, N = A.shape[0], B.shape[0]
    if C is None:
        C = torch.empty(M, N, device=A.device, dtype=dtype)
    P.oscars_gemm_i8_nt(A.data_ptr(), A.stride(0), sa.data_ptr(), B.data_ptr(), B.stride(0), sb.data_ptr(), C.data_ptr(),
                        C.stride(0), DT[dtype], M, N, K, bias_ptr=bias.data_ptr() if bias is not None else None, relu=relu,
                        stream=torch.cuda.current_stream().cuda_stream)
    return C


def check(C, A, B, sa, sb, K, bias=None, relu=False):
    acc = A[:, :K].double() @ B[:, :K].double().T   # exact: below 2^53
    prod = acc * sa.double()[:, None] * sb.double()
    want = prod if bias is None else prod + bias.double()
    tol = 3 * U * prod.abs() + U * want.abs()
    if relu:
        want = want.clamp(min=0)
    if C.dtype == torch.bfloat16:
        tol = tol + torch.finfo(torch.bfloat16).eps / 2 * want.abs()
    tol = tol * (1 + 2.0 ** -6) + 1e-38
    bad = (C.double() - want).abs() > tol
    assert not bad.any(), (bad.sum().item(), bad.nonzero()[0].tolist())


def scales(n, seed, dev):
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.rand(n, device=dev, generator=g) * 1e-2 + 1e-4


SIZES = [(1, 1, 1), (1, 1, 16), (1, 512, 784), (1, 10, 512), (2, 3, 5), (3, 130, 17), (4, 64, 64), (7, 1000, 129), (8, 128, 128),
         (15, 257, 100), (16, 256, 1024), (17, 63, 1025), (31, 100, 31), (33, 65, 2047), (63, 300, 96), (64, 64, 4096), (65, 200, 130),
         (100, 31, 33), (127, 129, 63), (128, 128, 128), (129, 257, 255), (200, 1, 300), (255, 256, 512), (256, 512, 784), (257, 255, 1040),
         (300, 1000, 77), (513, 384, 1100), (1000, 777, 640)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_matches_exact_sums(cuda_device, M, N, K, dtype):
    A, B = codes(M, K, 1, cuda_device, pad=16 * (M % 3)), codes(N, K, 2, cuda_device, pad=32 * (N % 2))
    sa, sb, bias = scales(M, 3, cuda_device), scales(N, 4, cuda_device), torch.randn(N, device=cuda_device)
    for b, relu in ((None, False), (bias, True)):
        check(product(A, B, sa, sb, K, dtype, b, relu), A, B, sa, sb, K, b, relu)


@pytest.mark.parametrize("M,N,K", [(2048, 2048, 1024), (4097, 1031, 530), (8192, 512, 784), (1, 8192, 8192), (40, 4096, 4096),
                                   (1024, 10, 512), (300, 5000, 3000)])
def test_large(cuda_device, M, N, K):
    A, B = codes(M, K, 1, cuda_device), codes(N, K, 2, cuda_device)
    sa, sb = scales(M, 3, cuda_device), scales(N, 4, cuda_device)
    check(product(A, B, sa, sb, K, torch.float32), A, B, sa, sb, K)


@pytest.mark.parametrize("M,N", [(1, 40), (5, 130), (40, 40), (200, 300)])
@pytest.mark.parametrize("K", [1023, 1024, 1025, 1041, 5000, 20000, 131071])
def test_sums_stay_exact(cuda_device, M, N, K):
    """All codes of one sign and the largest size: sums far past what fp32 holds exactly.  With unit scales the fp32
    result is the integer rounded once."""
    one_a, one_b = torch.ones(M, device=cuda_device), torch.ones(N, device=cuda_device)
    A, B = codes(M, K, 5, cuda_device, lo=125, hi=128), codes(N, K, 6, cuda_device, lo=-128, hi=-125)
    C = product(A, B, one_a, one_b, K, torch.float32)
    want = (A[:, :K].double() @ B[:, :K].double().T).float()
    assert torch.equal(C, want)
    A.fill_(-128)
    B.fill_(-128)
    assert (product(A, B, one_a, one_b, K, torch.float32) == float(K) * 16384.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K,shift,ldc", [(3, 70, 33, 1, 70), (40, 129, 64, 3, 131), (130, 64, 200, 0, 72), (129, 300, 96, 2, 301),
                                             (1, 33, 20, 5, 40), (260, 256, 128, 0, 264), (70, 256, 256, 0, 256)])
def test_c_anywhere(cuda_device, M, N, K, shift, ldc, dtype):
    """C at any alignment and row distance; what lies around and between its rows stays as it was."""
    A, B = codes(M, K, 1, cuda_device), codes(N, K, 2, cuda_device)
    sa, sb, bias = scales(M, 3, cuda_device), scales(N, 4, cuda_device), torch.randn(N, device=cuda_device)
    buf = torch.full((shift + M * ldc + 64,), 9.0, device=cuda_device, dtype=dtype)
    C = buf[shift:shift + M * ldc].view(M, ldc)[:, :N]
    product(A, B, sa, sb, K, dtype, bias, True, C)
    check(C, A, B, sa, sb, K, bias, True)
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask[shift:shift + M * ldc].view(M, ldc)[:, :N] = False
    assert (buf[mask] == 9.0).all()


@pytest.mark.parametrize("M", [1, 3, 20, 150, 300])
def test_special_scales(cuda_device, M):
    """Tokens whose scale is NaN, infinite or zero (as quantisation gives them) stay in their rows; ReLU keeps NaN."""
    N, K = 140, 100
    A, B = codes(M, K, 1, cuda_device), codes(N, K, 2, cuda_device)
    sa, sb = scales(M, 3, cuda_device), scales(N, 4, cuda_device)
    clean = product(A, B, sa, sb, K, torch.float32, relu=True).clone()
    for bad in (float("nan"), float("inf"), 0.0):
        s, Q = sa.clone(), A.clone()
        s[M // 2], Q[M // 2] = bad, 0
        C = product(Q, B, s, sb, K, torch.float32, relu=True)
        row = C[M // 2]
        assert (row == 0).all() if bad == 0.0 else torch.isnan(row).all()
        keep = torch.arange(M, device=cuda_device) != M // 2
        assert torch.equal(C[keep], clean[keep])


def test_no_tokens(cuda_device):
    P.oscars_gemm_i8_nt(0, 16, 0, 0, 16, 0, 0, 8, P.F32, 0, 8, 16)
    P.oscars_quantize_i8(0, 16, P.F32, 0, 16, 0, 16, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 512, 784), (20, 300, 500), (300, 512, 784), (1000, 1000, 1000)])
def test_repeats_on_streams_and_in_graphs(cuda_device, M, N, K, dtype):
    A, B = codes(M, K, 1, cuda_device), codes(N, K, 2, cuda_device)
    A2 = codes(M, K, 7, cuda_device)
    sa, sb = scales(M, 3, cuda_device), scales(N, 4, cuda_device)
    want, want2 = product(A, B, sa, sb, K, dtype).clone(), product(A2, B, sa, sb, K, dtype).clone()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(want) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, a in zip(streams, outs, (A, A2)):
            with torch.cuda.stream(s):
                product(a, B, sa, sb, K, dtype, C=o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want2)
    graph, s, inp, out = torch.cuda.CUDAGraph(), torch.cuda.Stream(), A.clone(), torch.empty_like(want)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        product(inp, B, sa, sb, K, dtype, C=out)
    for a, w in ((A2, want2), (A, want)):
        inp.copy_(a)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)


# ------------------------------------------------------------------ quantisation
def quantize(x, ldq=None, q=None):
    rows, cols = x.shape
    ldq = ldq or cols
    if q is None:
        q = torch.full((rows, ldq), 99, dtype=torch.int8, device=x.device)
    s = torch.full((rows,), -1.0, device=x.device)
    P.oscars_quantize_i8(x.data_ptr(), x.stride(0), DT[x.dtype], rows, cols, q.data_ptr(), q.stride(0), s.data_ptr(),
                         stream=torch.cuda.current_stream().cuda_stream)
    return q, s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 784, 0, 0), (3, 5, 11, 1), (7, 33, 0, 3), (64, 512, 0, 0), (5, 1000, 8, 0),
                                                 (2, 4096, 16, 0), (1000, 130, 2, 0), (4, 8192, 0, 0), (3, 20001, 7, 5), (2, 70000, 0, 0),
                                                 (8192, 784, 0, 0), (3, 1025, 0, 0), (7, 4096, 3, 1), (1, 3001, 0, 0), (5, 4097, 0, 2)])
def test_codes_equal_fp32_division(cuda_device, rows, cols, pad, shift, dtype):
    g = torch.Generator(device=cuda_device).manual_seed(rows + cols)
    buf = torch.randn(shift + rows * (cols + pad), device=cuda_device, generator=g).to(dtype)
    x = buf[shift:].view(rows, cols + pad)[:, :cols]
    ldq = cols + 3 * (pad > 0)
    q, s = quantize(x, ldq)
    f = x.float()
    want_s = (f.abs().amax(1).double() / 127.0).float()   # fp32 division (by a Python number torch multiplies instead)
    assert torch.equal(s, want_s)
    assert torch.equal(q[:, :cols], torch.round(f / want_s[:, None]).to(torch.int8))
    assert (q[:, cols:] == 99).all()


@pytest.mark.parametrize("cols", [1, 40, 1000, 30000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_special_rows(cuda_device, cols, dtype):
    """Zeros, infinities, NaN, the smallest and the largest numbers; the rows between are as they are alone."""
    x = torch.randn(9, cols, device=cuda_device).to(dtype)
    q0, s0 = quantize(x)
    x[1] = 0
    x[2, cols // 2] = float("inf")
    x[3, cols // 3] = float("nan")
    x[4, 0], x[4, cols - 1] = float("nan"), float("-inf")
    x[5] = 1e-45 if dtype == torch.float32 else 9.2e-41   # its scale underflows to zero, or nearly
    x[6] = torch.finfo(dtype).max
    q, s = quantize(x)
    for r in (0, 7, 8):
        assert torch.equal(q[r], q0[r]) and s[r] == s0[r]
    assert s[1] == 0 and (q[1] == 0).all()
    assert s[2] == float("inf") and (q[2] == 0).all()
    assert torch.isnan(s[3]) and (q[3] == 0).all()
    assert (q[4] == 0).all() and (torch.isnan(s[4]) if cols > 1 else s[4] == float("inf"))
    tiny = (x[5, 0].double() / 127).float().item()
    assert s[5] == tiny and (q[5] == (0 if tiny == 0 else 127)).all()
    assert (q[6] == 127).all()


def test_a_layer_of_quantised_tokens(cuda_device):
    """Quantise tokens and channels, multiply: each dequantised operand is off by at most half a step of its row's
    scale, which bounds the product against the unquantised one."""
    for M, N, K, dtype in [(1, 512, 784, torch.bfloat16), (70, 300, 500, torch.float32), (400, 257, 1030, torch.bfloat16)]:
        g = torch.Generator(device=cuda_device).manual_seed(K)
        x, W = torch.randn(M, K, device=cuda_device, generator=g).to(dtype), torch.randn(N, K, device=cuda_device, generator=g)
        ld = (K + 15) // 16 * 16
        A, sa = quantize(x, ld)
        B, sb = quantize(W, ld)
        C = product(A, B, sa, sb, K, torch.float32)
        check(C, A, B, sa, sb, K)
        want = x.double() @ W.double().T
        half_a, half_b = sa.double()[:, None] * 0.5001, sb.double()[:, None] * 0.5001
        tol = half_a * (W.double().abs().sum(1)) + (x.double().abs().sum(1)[:, None] + K * half_a) * half_b.T
        assert ((C.double() - want).abs() <= tol + 1e-4).all()
