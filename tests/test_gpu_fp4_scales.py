"""Products in 4 bits whose row scales, block scales and sums lie far apart: a finite result is finite and as exact as any, in every
kernel (one token, few, parts of K, results from registers and through shared memory) and in both formats.

The bounds are those of tests/test_gpu_fp4.py: with every intermediate result in fp32's normal numbers the row scales are two
roundings, relative to the result."""
import numpy as np
import pytest
import torch

import paper_2102_08550_gb300 as P
from tests.fp4_reference import BLOCK, Kept
from tests.test_gpu_fp4 import TYPES, check, product

pytestmark = pytest.mark.gpu
# M, N, K, distance of C's rows beyond N
SHAPES = [(1, 140, 200, 0), (3, 140, 200, 0), (4, 64, 70, 0), (40, 140, 200, 0), (16, 600, 3000, 0), (300, 300, 200, 0), (300, 300, 200, 1), (700, 640, 512, 0),
          (700, 640, 512, 1), (2100, 1300, 96, 0), (2100, 1300, 96, 1)]


def kept(rows, K, fmt, dev, seed, lo, hi, scales, positive=False):
    """Random codes (of 4 and 6 alone if positive) under block scales of bytes lo ... hi - 1, row scales given in turn."""
    rng = np.random.default_rng(seed)
    n = BLOCK[fmt]
    codes = rng.choice([6, 7], (rows, -(-K // 32) * 32)) if positive else rng.integers(0, 16, (rows, -(-K // 32) * 32))
    codes[:, K:] = 0
    blocks = -(-K // n)
    byte = np.zeros((rows, -(-blocks // 4) * 4), np.int64)
    byte[:, :blocks] = rng.integers(lo, hi, (rows, blocks))
    t = np.array([scales[i % len(scales)] for i in range(rows)], np.float32)
    return Kept(codes, byte, t, K, fmt, dev)


def out(M, N, more, dtype, dev):
    return torch.full((M, N + more), float("nan"), device=dev, dtype=dtype)[:, :N]


BELOW, ABOVE = float(np.nextafter(np.float32(2.0 ** -96), np.float32(0))), float(np.nextafter(np.float32(2.0 ** 64), np.float32(np.inf)))
# bytes of A's and of B's blocks, tokens' and channels' scales
MX = {"large sums, tokens just below 2^-96": ((181, 183), (181, 183), [2.0 ** -97, BELOW], [2.0 ** 60]),
      "large sums, channels small": ((177, 179), (177, 179), [2.0 ** 60], [2.0 ** -100]),
      "large sums, tokens small": ((177, 179), (177, 179), [2.0 ** -100, 2.0 ** -90], [2.0 ** 60, 3.0]),
      "small sums, channels large": ((67, 69), (67, 69), [2.0 ** -90, 2.0 ** -60], [2.0 ** 100, 2.0 ** 120]),
      "small sums, tokens large": ((67, 69), (67, 69), [2.0 ** 100, ABOVE], [2.0 ** -80, 1.0]),
      "plain rows among far ones": ((125, 129), (125, 129), [0.5, 2.0 ** -110, 3.0, 2.0 ** 80, 2.0 ** -140], [2.0 ** -20, 7.0, 2.0 ** 20])}
NV = {"tokens just above 2^64, channels at the smallest": ((1, 4), (1, 4), [2.0 ** 65, ABOVE, 2.0 ** 64], [1.1 * 2.0 ** -126]),
      "tokens just below 2^-96, channels at the largest": ((120, 127), (120, 127), [2.0 ** -97, BELOW, 2.0 ** -96], [2.0 ** 90]),
      "subnormal scales": ((60, 127), (60, 127), [2.0 ** 100, 2.0 ** 70], [3 * 2.0 ** -149, 2.0 ** -127]),
      "subnormal tokens": ((60, 127), (60, 127), [3 * 2.0 ** -149, 2.0 ** -127], [2.0 ** 100, 2.0 ** 70])}


@pytest.mark.parametrize("M,N,K,more", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt,what", [(P.MXFP4, w) for w in MX] + [(P.NVFP4, w) for w in NV])
def test_scales_far_apart(cuda_device, fmt, what, dtype, M, N, K, more):
    a, b, ta, tb = (MX if fmt == P.MXFP4 else NV)[what]
    A, B = kept(M, K, fmt, cuda_device, 1, *a, ta), kept(N, K, fmt, cuda_device, 2, *b, tb)
    C = product(A, B, dtype, C=out(M, N, more, dtype, cuda_device))
    assert torch.isfinite(C).all()
    check(C, A, B)
    bias = torch.full((N,), -3.0, device=cuda_device)
    C = product(A, B, dtype, bias, True, C=out(M, N, more, dtype, cuda_device))
    check(C, A, B, bias, True)


@pytest.mark.parametrize("M", [1, 2, 20, 300])
def test_sums_of_many_large_blocks(cuda_device, M):
    """4096 products of 4s and 6s under scales of 448: a sum of 2^34, which a token's scale below 2^-96 made 2^64 larger and a channel's
    of 2^127 took past fp32, where the result is 2^65."""
    A = kept(M, 4096, P.NVFP4, cuda_device, 1, 126, 127, [BELOW, 2.0 ** -97], positive=True)
    B = kept(200, 4096, P.NVFP4, cuda_device, 2, 126, 127, [2.0 ** 127], positive=True)
    C = product(A, B, torch.float32)
    assert torch.isfinite(C).all()
    check(C, A, B)


@pytest.mark.parametrize("fmt", [P.MXFP4, P.NVFP4])
@pytest.mark.parametrize("M,N,K,more", SHAPES)
def test_a_row_knows_nothing_of_its_neighbours(cuda_device, M, N, K, more, fmt):
    """Rows whose scales are far away, zero, infinite or no number leave the others' bits; their own are those of a call alone."""
    rng = np.random.default_rng(5)
    mid = (120, 134) if fmt == P.MXFP4 else (0, 127)
    plain = (rng.random(64) * 1e-2 + 1e-4).astype(np.float32).tolist()
    far = [s if i % 3 else f for i, (s, f) in enumerate(zip(plain, [2.0 ** -110, 2.0 ** 90, 0.0, float("inf"), float("nan"), 2.0 ** -140, 2.0 ** 70] * 10))]
    B = kept(N, K, fmt, cuda_device, 2, *mid, plain)
    A0, A1 = kept(M, K, fmt, cuda_device, 1, *mid, plain), kept(M, K, fmt, cuda_device, 1, *mid, far)
    C0, C1 = (product(A, B, torch.float32, C=out(M, N, more, torch.float32, cuda_device)) for A in (A0, A1))
    rows = torch.arange(M, device=cuda_device) % 64
    same = torch.tensor([a == b for a, b in zip(plain, far)], device=cuda_device)[rows]
    assert torch.equal(C0[same], C1[same])
    scale = torch.tensor(far, device=cuda_device, dtype=torch.float64)[rows]
    finite = torch.isfinite(scale)
    assert torch.isfinite(C1[finite]).all() and (C1[scale == 0] == 0).all() and torch.isnan(C1[torch.isnan(scale)]).all()
    inf = torch.isinf(scale)
    assert not torch.isfinite(C1[inf]).any()
    A1.row = torch.where(finite, scale, torch.ones_like(scale))
    C1[~finite] = C0[~finite]
    A1.row[~finite] = A0.row[~finite]
    check(C1, A1, B)
