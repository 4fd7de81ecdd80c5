"""Rows in 4 bits by their definition, in 64 bits with each documented rounding to fp32 made with numpy."""
import numpy as np
import torch

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {0: 32, 1: 16}   # MXFP4, NVFP4
# the non-negative finite e4m3 numbers, by their bytes
E4M3 = np.array([(b & 7) * 2.0 ** -9 if b < 8 else (8 + (b & 7)) * 2.0 ** ((b >> 3) - 10) for b in range(127)])


def nearest(v, table):
    """Index of the nearest entry of an ascending table, ties to the even index, past the end to the last."""
    v = np.minimum(v, table[-1])
    hi = np.clip(np.searchsorted(table, v, side="left"), 1, len(table) - 1)
    lo = hi - 1
    dl, dh = v - table[lo], table[hi] - v
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def encode(x, fmt):
    """(codes [rows][columns up to a multiple of 32], block bytes [rows][blocks up to a multiple of 4], row scales)."""
    x = x.detach().float().cpu().numpy()
    rows, cols = x.shape
    n = BLOCK[fmt]
    blocks = -(-cols // (4 * n)) * 4
    full = np.zeros((rows, blocks * n), np.float32)
    full[:, :cols] = x
    full = full.reshape(rows, blocks, n)
    row_bad = ~np.isfinite(full).all((1, 2))
    block_bad = ~np.isfinite(full).all(2)
    mag = np.abs(np.where(np.isfinite(full), full, 0)).astype(np.float64)
    m = mag.max(2)
    with np.errstate(all="ignore"):
        if fmt == 0:
            e = np.maximum(np.frexp(m)[1] - 3, -127)
            e = np.where(m == 0, -127, e)
            byte, t = e + 127, None
            codes = nearest(mag * np.exp2(-e.astype(np.float64))[:, :, None], VALUES)
            byte = np.where(block_bad, 255, byte)
            codes = np.where(block_bad[:, :, None], 0, codes)
        else:
            top = m.max(1)
            t = np.maximum((top / 2688.0).astype(np.float32), np.float32(2.0 ** -110))
            t = np.where(top == 0, np.float32(0), t).astype(np.float32)
            six = (t * np.float32(6)).astype(np.float32)
            g = np.where(t > 0, (np.float32(1) / six).astype(np.float32), np.float32(0))
            want = np.minimum((m.astype(np.float32) * g[:, None]).astype(np.float32), np.float32(448))
            byte = nearest(want.astype(np.float64), E4M3)
            s = (E4M3[byte].astype(np.float32) * t[:, None]).astype(np.float32)
            r = np.where(byte > 0, (np.float32(1) / s).astype(np.float32), np.float32(0))
            codes = nearest((mag.astype(np.float32) * r[:, :, None]).astype(np.float32).astype(np.float64), VALUES)
            byte = np.where(row_bad[:, None], 0, byte)
            codes = np.where(row_bad[:, None, None], 0, codes)
            nan = np.isnan(full).any((1, 2))
            t = np.where(nan, np.float32("nan"), np.where(row_bad, np.float32("inf"), t)).astype(np.float32)
    sign = np.signbit(full) & (codes > 0)
    codes = (codes + 8 * sign).reshape(rows, -1)[:, :-(-cols // 32) * 32]
    return codes, byte, t


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def tile_index(rows, blocks):
    """Byte of each (row, block) in the tiled scales; blocks is a multiple of 4."""
    i, j = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    return ((i // 128) * (blocks // 4) + j // 4) * 512 + (i % 32) * 16 + (i % 128) // 32 * 4 + j % 4


def matrix(codes, byte, cols, fmt):
    """Values without row scales, fp64."""
    v = np.where(codes >= 8, -1.0, 1.0) * VALUES[codes & 7]
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127)) if fmt == 0 else np.append(E4M3, np.nan)[byte]
    return v[:, :cols] * np.repeat(s, BLOCK[fmt], 1)[:, :cols]


class Kept:
    """A matrix in 4 bits on the device, from random codes and bytes or from values."""

    def __init__(self, codes, byte, t, cols, fmt, dev, pad=0):
        rows = codes.shape[0]
        self.rows, self.cols, self.fmt = rows, cols, fmt
        q = np.full((rows, codes.shape[1] // 2 + pad), 0x5A, np.uint8)   # bytes behind the last group of 32 are anything
        q[:, :codes.shape[1] // 2] = pack(codes)
        s = np.full(-(-rows // 128) * (byte.shape[1] // 4) * 512, 0xFF, np.uint8)   # rows behind the last too
        s[tile_index(rows, byte.shape[1])] = byte
        self.q, self.s = torch.from_numpy(q).to(dev), torch.from_numpy(s).to(dev)
        self.t = None if t is None else torch.from_numpy(t).to(dev)
        self.values = torch.from_numpy(matrix(codes, byte, cols, fmt)).to(dev)
        self.row = self.t.double() if t is not None else torch.ones(rows, dtype=torch.float64, device=dev)

    @staticmethod
    def random(rows, cols, fmt, dev, seed, pad=0, lo=None, hi=None, row_scales=None):
        rng = np.random.default_rng(seed)
        n = BLOCK[fmt]
        codes = rng.integers(0, 16, (rows, -(-cols // 32) * 32))
        codes[:, cols:] = 0
        blocks = -(-cols // n)
        byte = np.zeros((rows, -(-blocks // 4) * 4), np.int64)
        lo, hi = (lo, hi) if lo is not None else ((118, 136) if fmt == 0 else (0, 127))
        byte[:, :blocks] = rng.integers(lo, hi, (rows, blocks))
        row_scales = fmt == 1 if row_scales is None else row_scales
        t = (rng.random(rows) * 1e-2 + 1e-4).astype(np.float32) if row_scales else None
        return Kept(codes, byte, t, cols, fmt, dev, pad)
