"""Rows in 4 bits against their definition bit by bit, and their products against 64-bit sums.

Tolerance of a product, element by element.  Products of codes and their sums over a block are exact; what is added up in
fp32 are at most K / 16 block sums, each addition (and each scaling of a block's sum) off by at most a whole step of fp32,
2^-23, of what has come together so far, which is at most S = sum |A| |B|.  The row scales and the bias are three roundings of
the result more, and the result's own rounding is half a step of its type."""
import numpy as np
import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.fp4_reference import BLOCK, Kept, encode, matrix, pack, tile_index

pytestmark = pytest.mark.gpu
DT = {torch.float32: P.F32, torch.bfloat16: P.BF16}
TYPES = [torch.float32, torch.bfloat16]
FORMATS = [P.MXFP4, P.NVFP4]


def stream():
    return torch.cuda.current_stream().cuda_stream


def product(A, B, dtype, bias=None, relu=False, C=None):
    M, N, K = A.rows, B.rows, A.cols
    if C is None:
        C = torch.full((M, N), float("nan"), device=A.q.device, dtype=dtype)
    P.oscars_gemm_fp4_nt(A.q.data_ptr(), A.q.stride(0), A.s.data_ptr(), B.q.data_ptr(), B.q.stride(0), B.s.data_ptr(), A.fmt, C.data_ptr(),
                         C.stride(0), DT[dtype], M, N, K, row_scale_a_ptr=A.t.data_ptr() if A.t is not None else None,
                         row_scale_b_ptr=B.t.data_ptr() if B.t is not None else None,
                         bias_ptr=bias.data_ptr() if bias is not None else None, relu=relu, stream=stream())
    return C


def check(C, A, B, bias=None, relu=False):
    scale = A.row[:, None] * B.row
    prod = A.values @ B.values.T * scale
    S = A.values.abs() @ B.values.abs().T * scale
    want = prod if bias is None else prod + bias.double()
    tol = 2.0 ** -23 * (A.cols / 16 + 2) * S + 2.0 ** -24 * (3 * prod.abs() + want.abs())
    if relu:
        want = want.clamp(min=0)
    if C.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + torch.finfo(torch.bfloat16).eps / 2 * want.abs()
    bad = ~((C.double() - want).abs() <= tol * (1 + 2.0 ** -6) + 1e-38)
    assert not bad.any(), (bad.sum().item(), bad.nonzero()[0].tolist())


SIZES = [(1, 1, 1), (1, 1, 16), (1, 512, 784), (1, 10, 512), (2, 3, 5), (3, 130, 17), (4, 64, 64), (7, 1000, 129), (8, 128, 128),
         (15, 257, 100), (16, 256, 1024), (17, 63, 1025), (31, 100, 31), (33, 65, 2047), (63, 300, 96), (64, 64, 4096), (65, 200, 130),
         (100, 31, 33), (127, 129, 63), (128, 128, 128), (129, 257, 255), (200, 1, 300), (255, 256, 512), (256, 512, 784), (257, 255, 1040),
         (300, 1000, 77), (513, 384, 1100), (1000, 777, 640), (96, 2000, 260), (161, 1300, 320)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_matches_64_bit_sums(cuda_device, M, N, K, dtype, fmt):
    A = Kept.random(M, K, fmt, cuda_device, 1, pad=16 * (M % 3))
    B = Kept.random(N, K, fmt, cuda_device, 2, pad=32 * (N % 2))
    bias = torch.randn(N, device=cuda_device)
    for b, relu in ((None, False), (bias, True)):
        check(product(A, B, dtype, b, relu), A, B, b, relu)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(2048, 2048, 1024), (4097, 1031, 530), (8192, 512, 784), (1, 8192, 8192), (40, 4096, 4096),
                                   (1024, 10, 512), (300, 5000, 3000), (2500, 3100, 96), (16, 4096, 4096), (5, 300, 20000)])
def test_large(cuda_device, M, N, K, fmt):
    A, B = Kept.random(M, K, fmt, cuda_device, 1), Kept.random(N, K, fmt, cuda_device, 2)
    check(product(A, B, torch.float32), A, B)
    check(product(A, B, torch.bfloat16), A, B)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (3, 130, 300), (40, 257, 1024), (300, 300, 200)])
def test_row_scales_are_optional(cuda_device, M, N, K, fmt):
    for ra, rb in ((False, False), (True, False), (False, True), (True, True)):
        A = Kept.random(M, K, fmt, cuda_device, 1, row_scales=ra)
        B = Kept.random(N, K, fmt, cuda_device, 2, row_scales=rb)
        check(product(A, B, torch.float32), A, B)


@pytest.mark.parametrize("M,N,K", [(1, 50, 96), (20, 140, 200), (200, 300, 160)])
def test_powers_of_two_over_their_range(cuda_device, M, N, K):
    """MX scales from 2^-127 to 2^125 on one side against their opposites on the other."""
    for lo in (0, 40, 180, 245):
        A = Kept.random(M, K, P.MXFP4, cuda_device, 1, lo=lo, hi=lo + 6)
        other = min(254 - lo, 246)
        B = Kept.random(N, K, P.MXFP4, cuda_device, 2, lo=other, hi=other + 6)
        check(product(A, B, torch.float32), A, B)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K,shift,ldc", [(3, 70, 33, 1, 70), (40, 129, 64, 3, 131), (130, 64, 200, 0, 72), (129, 300, 96, 2, 301),
                                             (1, 33, 20, 5, 40), (260, 256, 128, 0, 264), (70, 256, 256, 0, 256), (600, 520, 64, 1, 523)])
def test_c_anywhere(cuda_device, M, N, K, shift, ldc, dtype, fmt):
    """C at any alignment and row distance; what lies around and between its rows stays as it was."""
    A, B = Kept.random(M, K, fmt, cuda_device, 1), Kept.random(N, K, fmt, cuda_device, 2)
    bias = torch.randn(N, device=cuda_device)
    buf = torch.full((shift + M * ldc + 64,), 9.0, device=cuda_device, dtype=dtype)
    C = buf[shift:shift + M * ldc].view(M, ldc)[:, :N]
    product(A, B, dtype, bias, True, C)
    check(C, A, B, bias, True)
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask[shift:shift + M * ldc].view(M, ldc)[:, :N] = False
    assert (buf[mask] == 9.0).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [1, 3, 20, 150, 300])
def test_special_scales_stay_in_their_rows(cuda_device, M, fmt):
    """A token with a NaN block (MX) or a NaN or infinite row (NV), as quantisation writes them; ReLU keeps NaN."""
    N, K = 140, 100
    x, W = torch.randn(M, K, device=cuda_device), torch.randn(N, K, device=cuda_device)
    kept = lambda v: Kept(*encode(v, fmt), K, fmt, cuda_device)
    B = kept(W)
    clean = product(kept(x), B, torch.float32, relu=True)
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[M // 2, K // 3] = bad
        C = product(kept(y), B, torch.float32, relu=True)
        assert torch.isnan(C[M // 2]).all()
        keep = torch.arange(M, device=cuda_device) != M // 2
        assert torch.equal(C[keep], clean[keep])
    y = x.clone()
    y[M // 2] = 0
    assert (product(kept(y), B, torch.float32)[M // 2] == 0).all()


@pytest.mark.parametrize("M", [1, 4, 40, 300])
def test_row_scales_at_the_ends_of_fp32(cuda_device, M):
    """Tokens of 1e37 against channels of 1e-30, and the other way round: only the result may leave fp32."""
    N, K = 140, 200
    x, W = torch.randn(M, K, device=cuda_device), torch.randn(N, K, device=cuda_device)
    for sx, sw in ((1e37, 1e-30), (1e-30, 1e37), (1e37, 1e-3), (3e-33, 1.0)):
        A, B = (Kept(*encode(v, P.NVFP4), K, P.NVFP4, cuda_device) for v in (x * sx, W * sw))
        C = product(A, B, torch.float32)
        assert torch.isfinite(C).all()
        check(C, A, B)


def test_no_rows(cuda_device):
    P.oscars_gemm_fp4_nt(0, 16, 0, 0, 16, 0, P.MXFP4, 0, 8, P.F32, 0, 8, 16)
    P.oscars_quantize_fp4(0, 16, P.F32, 0, 16, P.MXFP4, 0, 16, 0)
    P.oscars_dequantize_fp4(0, 16, 0, 0, P.NVFP4, 0, 16, 0, 16, P.F32)
    assert P.oscars_fp4_scale_bytes(0, 16, P.NVFP4) == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 512, 784), (20, 300, 500), (300, 512, 784), (1000, 1000, 1000), (16, 4096, 1024), (700, 2600, 512)])
def test_repeats_on_streams_and_in_graphs(cuda_device, M, N, K, dtype, fmt):
    A, B, A2 = (Kept.random(r, K, fmt, cuda_device, i) for r, i in ((M, 1), (N, 2), (M, 7)))
    want, want2 = product(A, B, dtype).clone(), product(A2, B, dtype).clone()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(want) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, a in zip(streams, outs, (A, A2)):
            with torch.cuda.stream(s):
                product(a, B, dtype, C=o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want2)
    graph, s, out = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.empty_like(want)
    inp = Kept.random(M, K, fmt, cuda_device, 1)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        product(inp, B, dtype, C=out)
    for a, w in ((A2, want2), (A, want)):
        inp.q.copy_(a.q)
        inp.s.copy_(a.s)
        if inp.t is not None:
            inp.t.copy_(a.t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)


# ------------------------------------------------------------------ quantisation
def quantize(x, fmt, ldq=None):
    rows, cols = x.shape
    ldq = ldq or (cols + 31) // 32 * 16
    q = torch.full((rows, ldq), 0x5A, dtype=torch.uint8, device=x.device)
    s = torch.full((P.oscars_fp4_scale_bytes(rows, cols, fmt),), 0x5A, dtype=torch.uint8, device=x.device)
    t = torch.full((rows,), -1.0, device=x.device) if fmt == P.NVFP4 else None
    P.oscars_quantize_fp4(x.data_ptr(), x.stride(0), DT[x.dtype], rows, cols, fmt, q.data_ptr(), ldq, s.data_ptr(),
                          t.data_ptr() if t is not None else None, stream=stream())
    return q, s, t


def dequantize(q, s, t, cols, fmt, dtype, x=None):
    rows = q.shape[0]
    if x is None:
        x = torch.full((rows, cols), 7.0, device=q.device, dtype=dtype)
    P.oscars_dequantize_fp4(q.data_ptr(), q.stride(0), s.data_ptr(), t.data_ptr() if t is not None else None, fmt, rows, cols, x.data_ptr(),
                            x.stride(0), DT[dtype], stream=stream())
    return x


def check_codes(x, fmt, q, s, t):
    rows, cols = x.shape
    codes, byte, row = encode(x, fmt)
    got, used = q.cpu().numpy(), codes.shape[1] // 2
    low, high = got[:, :used] & 15, got[:, :used] >> 4
    mine = np.stack([low, high], 2).reshape(rows, -1)
    same = (mine == codes) | ((mine == 8) & (codes == 0))   # a small negative value may be -0
    assert same.all(), np.argwhere(~same)[:3]
    assert (got[:, used:] == 0x5A).all()
    index, flat = tile_index(rows, byte.shape[1]), s.cpu().numpy()
    assert (flat[index] == byte).all(), np.argwhere(flat[index] != byte)[:3]
    rest = np.ones(flat.shape, bool)
    rest[index] = False
    assert (flat[rest] == 0x5A).all()
    if fmt == P.NVFP4:
        assert np.array_equal(t.cpu().numpy(), row, equal_nan=True)
    return codes, byte, row


SHAPES = [(1, 1, 0, 0), (1, 784, 0, 0), (3, 5, 11, 1), (7, 33, 0, 3), (64, 512, 0, 0), (5, 1000, 8, 0), (2, 4096, 16, 0), (300, 130, 2, 0),
          (4, 8192, 0, 0), (3, 20001, 7, 5), (2, 70000, 0, 0), (1024, 784, 0, 0), (3, 1025, 0, 0), (7, 4096, 3, 1), (1, 3001, 0, 0),
          (5, 4097, 0, 2), (129, 64, 0, 0), (130, 63, 1, 0), (9, 127, 0, 0), (9, 129, 0, 0), (33, 16, 0, 0), (2, 17, 0, 0), (2, 31, 1, 1)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,shift", SHAPES)
def test_codes_by_definition(cuda_device, rows, cols, pad, shift, dtype, fmt):
    g = torch.Generator(device=cuda_device).manual_seed(rows + cols)
    buf = torch.randn(shift + rows * (cols + pad), device=cuda_device, generator=g)
    buf *= torch.exp(2 * torch.randn(buf.shape, device=cuda_device, generator=g))
    buf = buf.to(dtype)
    x = buf[shift:].view(rows, cols + pad)[:, :cols]
    q, s, t = quantize(x, fmt, (cols + 31) // 32 * 16 + 32 * (pad > 0))
    codes, byte, row = check_codes(x, fmt, q, s, t)
    # and back: the exact value rounded to fp32, times the row's scale
    for out in TYPES:
        v = torch.from_numpy(matrix(codes, byte, cols, fmt).astype(np.float32)).to(cuda_device)
        want = (v if t is None else v * t[:, None]).to(out)
        room = torch.full((shift + rows * (cols + pad) + 8,), 7.0, device=cuda_device, dtype=out)
        y = room[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        dequantize(q, s, t, cols, fmt, out, y)
        assert torch.equal(y, want)
        assert (room[:shift] == 7).all() and (room[shift:shift + rows * (cols + pad)].view(rows, -1)[:, cols:] == 7).all() and (room[-8:] == 7).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 40, 1000, 30000])
def test_special_rows(cuda_device, cols, dtype, fmt):
    """Zeros, infinities, NaN, the smallest and the largest numbers, ties."""
    x = torch.randn(10, cols, device=cuda_device).to(dtype)
    x[1] = 0
    x[2, cols // 2] = float("inf")
    x[3, cols // 3] = float("nan")
    x[4, 0], x[4, cols - 1] = float("nan"), float("-inf")
    x[5] = 1e-45 if dtype == torch.float32 else 9.2e-41
    x[6] = torch.finfo(dtype).max
    x[7] = torch.finfo(dtype).tiny
    ties = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -2.5, -3.5, -5.0, 0.0, 0.5, 3.0], device=cuda_device)
    x[8] = ties.repeat(cols // 16 + 1)[:cols].to(dtype)
    x[9, ::2] = torch.finfo(dtype).max
    x[9, 1::2] = -torch.finfo(dtype).max
    q, s, t = quantize(x, fmt)
    check_codes(x, fmt, q, s, t)
    y = dequantize(q, s, t, cols, fmt, torch.float32)
    assert torch.isnan(y[3, cols // 3]) and torch.isnan(y[2, cols // 2])
    assert (y[1] == 0).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_scale_back(cuda_device, fmt):
    """Every byte a scale can be, with every code."""
    n = BLOCK[fmt]
    blocks = 128
    byte = np.arange(256 if fmt == 0 else 128).reshape(-1, blocks)
    rows = byte.shape[0]
    codes = np.tile(np.arange(16), rows * blocks * n // 16).reshape(rows, -1)
    K = Kept(codes, byte, None, blocks * n, fmt, cuda_device)
    y = dequantize(K.q, K.s, None, blocks * n, fmt, torch.float32)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(matrix(codes, byte, blocks * n, fmt).astype(np.float32)).to(cuda_device)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.nan_to_num(y, 0.0), torch.nan_to_num(want, 0.0))
    t = torch.full((rows,), 3.0, device=cuda_device)
    y = dequantize(K.q, K.s, t, blocks * n, fmt, torch.float32)
    assert torch.equal(torch.nan_to_num(y, 0.0), torch.nan_to_num(want * 3.0, 0.0))
