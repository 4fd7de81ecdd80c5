"""Timed cases of layers kept in 4 bits and of the layer norm in front of them.

* ``codes``: rows become 4-bit codes with a scale for each block
  (``oscars_quantize_fp4``) and are unpacked again (``oscars_dequantize_fp4``): what
  a weight or a pushed delta is worth in 4 bits;
* ``product``: a product of operands in 4 bits, with bias and ReLU in its epilogue
  (``oscars_gemm_fp4_nt``);
* ``layer``: tokens in bf16 or fp32 are quantised and multiplied with a weight
  that is kept in 4 bits;
* ``norm``: layer norm's forward pass (``oscars_layer_norm``), with the statistics
  that training keeps;
* ``grad``: its backward pass with the gradients of its parameters
  (``oscars_layer_norm_backward``), for one model or for groups of rows that have
  parameters of their own (workers' replicas).

Two formats: ``mx`` (blocks of 32 with a power of two) and ``nv`` (blocks of 16
with an 8-bit scale, and an fp32 scale for each row).  Where ``own`` is false,
``run`` computes the same in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
BLOCK = {"mx": 32, "nv": 16}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one sample in front of the headline model's hidden layer: latency alone
        {"name": "norm-1x512-f32", "kind": "norm", "groups": 1, "rows": 1, "cols": 512, "dtype": "f32", "pad": 0},
        # a long prompt's activations, or a large evaluation batch's
        {"name": "norm-8192x4096-bf16", "kind": "norm", "groups": 1, "rows": 8192, "cols": 4096, "dtype": "bf16", "pad": 0},
        # one local step of sixteen workers: a mini-batch of 64 each, parameters of their own
        {"name": "grad-16x64x512-f32", "kind": "grad", "groups": 16, "rows": 64, "cols": 512, "dtype": "f32", "pad": 0},
        # odd rows and columns, rows further apart than their width
        {"name": "grad-1003x777-f32", "kind": "grad", "groups": 1, "rows": 1003, "cols": 777, "dtype": "f32", "pad": 6},
        # a training step of a large model
        {"name": "grad-16384x4096-bf16", "kind": "grad", "groups": 1, "rows": 16384, "cols": 4096, "dtype": "bf16", "pad": 0},
        # a ragged weight through 4 bits and back, blocks that end inside a row's last 32
        {"name": "codes-1001x333-mx-f32", "kind": "codes", "rows": 1001, "cols": 333, "format": "mx", "dtype": "f32", "pad": 6},
        # the tokens of a long prompt, or a large projection's weight
        {"name": "codes-8192x4096-nv-bf16", "kind": "codes", "rows": 8192, "cols": 4096, "format": "nv", "dtype": "bf16", "pad": 0},
        # a single sample through the headline model's hidden layer
        {"name": "layer-1x512x784-nv-bf16", "kind": "layer", "M": 1, "N": 512, "K": 784, "format": "nv", "dtype": "bf16", "bias": True, "relu": True},
        # sixteen samples through a large projection: the weights' bytes are what counts
        {"name": "layer-16x4096x4096-nv-bf16", "kind": "layer", "M": 16, "N": 4096, "K": 4096, "format": "nv", "dtype": "bf16", "bias": False, "relu": False},
        # the held-out set of the headline model through its hidden layer
        {"name": "layer-8192x512x784-mx-f32", "kind": "layer", "M": 8192, "N": 512, "K": 784, "format": "mx", "dtype": "f32", "bias": True, "relu": True},
        # ragged operands already in 4 bits, fp32 out
        {"name": "product-777x1003x1537-mx-f32", "kind": "product", "M": 777, "N": 1003, "K": 1537, "format": "mx", "dtype": "f32", "bias": True, "relu": False},
        # a long prompt or a large evaluation batch through a large projection
        {"name": "product-8192x4096x4096-nv-bf16", "kind": "product", "M": 8192, "N": 4096, "K": 4096, "format": "nv", "dtype": "bf16", "bias": False, "relu": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 200)


def draw(rng):
    """One more case of the same ranges, no more work than the largest listed one."""
    largest = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= largest:
            return case


def _draw(rng):
    kind = rng.choice(["codes", "product", "layer", "norm", "grad"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("norm", "grad"):
        groups = rng.choice([1, 1, _log_int(rng, 1, 32)])
        return {"kind": kind, "groups": groups, "rows": _log_int(rng, 1, 16384 // groups), "cols": _log_int(rng, 8, 8192),
                "dtype": dtype, "pad": rng.choice([0, 0, 0, 1, 24])}
    fmt = rng.choice(["mx", "nv"])
    if kind == "codes":
        return {"kind": kind, "rows": _log_int(rng, 1, 8192), "cols": _log_int(rng, 1, 8192), "format": fmt, "dtype": dtype,
                "pad": rng.choice([0, 0, 0, 1, 24])}
    return {"kind": kind, "M": _log_int(rng, 1, 8192), "N": _log_int(rng, 1, 8192), "K": _log_int(rng, 1, 8192), "format": fmt,
            "dtype": dtype, "bias": rng.random() < 0.5, "relu": rng.random() < 0.5}


def _coded(rows, cols, fmt):
    """Bytes of a matrix in 4 bits: codes, block scales, row scales."""
    return rows * (cols / 2 + cols / BLOCK[fmt] + (4 if fmt == "nv" else 0))


def work(case):
    k = case["kind"]
    size = 4 if case["dtype"] == "f32" else 2
    if k in ("norm", "grad"):
        n, rows, params = case["groups"] * case["rows"] * case["cols"], case["groups"] * case["rows"], case["groups"] * case["cols"]
        if k == "norm":   # x in, y out, gamma, beta, mean, rstd
            return {"bytes": 2 * n * size + 8 * params + 8 * rows, "flops": 8 * n}
        # dy and x in, dx out, gamma in, its gradient and beta's out
        return {"bytes": 3 * n * size + 12 * params + 8 * rows, "flops": 14 * n}
    if k == "codes":   # x in, codes out and in, values out
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * size + int(2 * _coded(case["rows"], case["cols"], case["format"])), "flops": 4 * n}
    M, N, K = case["M"], case["N"], case["K"]
    left = M * K * size if k == "layer" else _coded(M, K, case["format"])
    return {"bytes": int(left + _coded(N, K, case["format"])) + (4 * N if case["bias"] else 0) + M * N * size, "flops": 2 * M * N * K}


# ------------------------------------------------------------------ 4 bits
def _values(device):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=device)


def _nearest(u):
    """Index of the nearest of the eight magnitudes of a 4-bit code, ties to the even one."""
    return ((u > 0.25).to(torch.uint8) + (u >= 0.75) + (u > 1.25) + (u >= 1.75) + (u > 2.5) + (u >= 3.5) + (u > 5.0))


def _encode(x, fmt):
    """(codes 0..15 [rows][blocks][block], scales' bytes [rows][blocks], row scales or None) of finite fp32 rows."""
    rows, cols = x.shape
    n = BLOCK[fmt]
    x = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, n)
    m = x.abs().amax(2)
    if fmt == "mx":
        e = torch.clamp(torch.frexp(m)[1] - 3, min=-127)   # floor(log2 m) - 2
        e = torch.where(m == 0, torch.full_like(e, -127), e)
        u = (x.abs().double() * torch.exp2(-e.double()).unsqueeze(2)).float()
        byte, t = (e + 127).to(torch.uint8), None
    else:
        top = m.amax(1)
        t = torch.clamp(top / torch.full_like(top, 2688.0), min=2.0 ** -110)
        t = torch.where(top == 0, torch.zeros_like(t), t)
        b = torch.clamp(m * torch.where(top == 0, top, 1.0 / (t * 6.0)).unsqueeze(1), max=448.0).to(torch.float8_e4m3fn)
        s = b.float() * t.unsqueeze(1)
        u = x.abs() * torch.where(s == 0, s, 1.0 / s).unsqueeze(2)
        byte = b.view(torch.uint8)
    return _nearest(u) + (x < 0) * 8, byte, t


def _pack(codes, byte, rows):
    """Codes two a byte, scales in tiles of 128 rows x 4 blocks: row r of a tile at byte (r % 32) 16 + (r / 32) 4."""
    flat = codes.reshape(rows, -1)
    q = flat[:, 0::2] | (flat[:, 1::2] << 4)
    tiles = torch.nn.functional.pad(byte, (0, -byte.shape[1] % 4, 0, -rows % 128))
    s = tiles.reshape(tiles.shape[0] // 128, 4, 32, -1, 4).permute(0, 3, 2, 1, 4).contiguous()
    return q.contiguous(), s.reshape(-1)


def _unpack(q, s, rows, cols, fmt):
    """fp32 values without the row scale, from codes and tiled scales."""
    blocks = (cols + BLOCK[fmt] - 1) // BLOCK[fmt]
    kt = (blocks + 3) // 4
    byte = s.reshape(-1, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, kt * 4)[:rows, :blocks]
    if fmt == "mx":
        scale = torch.exp2(byte.double() - 127.0).float()
    else:
        scale = byte.contiguous().view(torch.float8_e4m3fn).float()
    codes = torch.stack([q & 15, q >> 4], 2).reshape(rows, -1)[:, :cols].int()
    v = _values(q.device)[codes & 7] * (1.0 - 2.0 * (codes >> 3))
    return v * scale.repeat_interleave(BLOCK[fmt], 1)[:, :cols]


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _activations(g, rows, cols):
    """Gaussian with a few wide channels, rows of different sizes."""
    x = torch.randn(rows, cols, device=DEV, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, device=DEV, generator=g))
    x *= 1.0 + 4.0 * (torch.rand(cols, device=DEV, generator=g) < 0.02)
    return x


def _apart(t, pad):
    """The matrix with its rows `pad` elements further apart than its width."""
    buf = torch.zeros(t.shape[0], t.shape[1] + pad, device=DEV, dtype=t.dtype)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def prepare(case, seed):
    g = _gen(seed)
    k = case["kind"]
    if k in ("norm", "grad"):
        n, r, c = case["groups"], case["rows"], case["cols"]
        x = _activations(g, n * r, c) + 0.5 * torch.randn(n * r, 1, device=DEV, generator=g)
        st = {"case": case, "x": _apart(x.to(_dtype(case)), case["pad"]), "out": torch.empty(n * r, c, device=DEV, dtype=_dtype(case)),
              "gamma": 1.0 + 0.2 * torch.randn(n, c, device=DEV, generator=g), "beta": 0.1 * torch.randn(n, c, device=DEV, generator=g)}
        if k == "norm":
            st["mean"], st["rstd"] = torch.empty(n * r, device=DEV), torch.empty(n * r, device=DEV)
            return st
        # what the forward pass left
        x = st["x"].double()
        mean = x.mean(1)
        st["mean"], st["rstd"] = mean.float(), (((x - mean[:, None]) ** 2).mean(1) + EPS).rsqrt().float()
        dy = 1e-3 * torch.randn(n * r, c, device=DEV, generator=g) * torch.exp(0.5 * torch.randn(n * r, 1, device=DEV, generator=g))
        st["dy"] = _apart(dy.to(_dtype(case)), case["pad"])
        st["dgamma"], st["dbeta"] = torch.empty(n, c, device=DEV), torch.empty(n, c, device=DEV)
        return st
    fmt = case["format"]

    def in_4_bits(x):   # the checkpoint's weights, or tokens that the layer before left in 4 bits
        codes, byte, t = _encode(x, fmt)
        return (*_pack(codes, byte, x.shape[0]), t)

    def room(rows, cols):
        return (torch.zeros(rows, (cols + 31) // 32 * 16, device=DEV, dtype=torch.uint8),
                torch.zeros((rows + 127) // 128 * (((cols + BLOCK[fmt] - 1) // BLOCK[fmt] + 3) // 4) * 512, device=DEV, dtype=torch.uint8),
                torch.zeros(rows, device=DEV) if fmt == "nv" else None)

    if k == "codes":
        r, c = case["rows"], case["cols"]
        x = _activations(g, r, c).to(_dtype(case))
        return {"case": case, "x": _apart(x, case["pad"]), "A": room(r, c), "out": torch.empty(r, c, device=DEV, dtype=_dtype(case))}
    M, N, K = case["M"], case["N"], case["K"]
    st = {"case": case, "C": torch.empty(M, N, device=DEV, dtype=_dtype(case)),
          "bias": torch.randn(N, device=DEV, generator=g) * 0.1 if case["bias"] else None,
          "B": in_4_bits(torch.randn(N, K, device=DEV, generator=g) / math.sqrt(K))}
    x = _activations(g, M, K)
    if k == "layer":
        st["x"], st["A"] = x.to(_dtype(case)), room(M, K)
    else:
        st["A"] = in_4_bits(x)
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _decoded(codes, byte, t, rows, cols, fmt):
    """fp32 values, without the row scale, of codes that are still apart."""
    scale = torch.exp2(byte.double() - 127.0).float() if fmt == "mx" else byte.view(torch.float8_e4m3fn).float()
    v = _values(codes.device)[(codes & 7).int()] * (1.0 - 2.0 * (codes >> 3).float())
    return (v * scale.unsqueeze(2)).reshape(rows, -1)[:, :cols]


def _run_plain(state):
    case = state["case"]
    k = case["kind"]
    if k in ("norm", "grad"):
        n, r, c = case["groups"], case["rows"], case["cols"]
        x = state["x"].float().reshape(n, r, c)
        gamma, beta = state["gamma"].unsqueeze(1), state["beta"].unsqueeze(1)
        if k == "norm":
            mean = x.mean(2, keepdim=True)
            d = x - mean
            rstd = 1.0 / ((d * d).mean(2, keepdim=True) + EPS).sqrt()
            y = d * rstd * gamma + beta
            return {"y": y.to(_dtype(case)).reshape(n * r, c), "mean": mean.reshape(-1), "rstd": rstd.reshape(-1)}
        dy = state["dy"].float().reshape(n, r, c)
        rstd = state["rstd"].reshape(n, r, 1)
        xh = (x - state["mean"].reshape(n, r, 1)) * rstd
        gr = dy * gamma
        dx = rstd * (gr - gr.mean(2, keepdim=True) - xh * (gr * xh).mean(2, keepdim=True))
        return {"dx": dx.to(_dtype(case)).reshape(n * r, c), "dgamma": (dy * xh).sum(1), "dbeta": dy.sum(1)}
    fmt = case["format"]
    if k == "codes":
        r, c = case["rows"], case["cols"]
        codes, byte, t = _encode(state["x"].float(), fmt)
        v = _decoded(codes, byte, t, r, c, fmt)
        return (v if t is None else v * t.unsqueeze(1)).to(_dtype(case))
    M, N, K = case["M"], case["N"], case["K"]
    if k == "layer":
        codes, byte, ta = _encode(state["x"].float(), fmt)
        A = _decoded(codes, byte, ta, M, K, fmt)
    else:
        q, s, ta = state["A"]
        A = _unpack(q, s, M, K, fmt)
    q, s, tb = state["B"]
    y = A @ _unpack(q, s, N, K, fmt).T
    if fmt == "nv":
        y = y * ta.unsqueeze(1) * tb
    if case["bias"]:
        y = y + state["bias"]
    if case["relu"]:
        y = torch.relu(y)
    return y.to(_dtype(case))


def _run_own(state):
    import paper_2102_08550_gb300 as lib

    case = state["case"]
    k = case["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    dt = lib.BF16 if case["dtype"] == "bf16" else lib.F32
    if k in ("norm", "grad"):
        n, r, c = case["groups"], case["rows"], case["cols"]
        x, out, gamma, beta, mean, rstd = (state[i] for i in ("x", "out", "gamma", "beta", "mean", "rstd"))
        if k == "norm":
            lib.oscars_layer_norm(x.data_ptr(), x.stride(0), gamma.data_ptr(), beta.data_ptr(), c, out.data_ptr(), c, dt, n, r, c, EPS,
                                  mean_ptr=mean.data_ptr(), rstd_ptr=rstd.data_ptr(), stream=stream)
            return {"y": out, "mean": mean, "rstd": rstd}
        if "ws" not in state:   # kept by the program, as its buffers are
            state["ws"] = torch.empty(lib.oscars_layer_norm_backward_workspace(n, r, c), device=DEV, dtype=torch.uint8)
        dy, ws, dgamma, dbeta = state["dy"], state["ws"], state["dgamma"], state["dbeta"]
        lib.oscars_layer_norm_backward(dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), gamma.data_ptr(), c, mean.data_ptr(),
                                       rstd.data_ptr(), out.data_ptr(), c, dgamma.data_ptr(), dbeta.data_ptr(), c, dt, n, r, c,
                                       ws.data_ptr(), ws.numel(), stream=stream)
        return {"dx": out, "dgamma": dgamma, "dbeta": dbeta}
    fmt = lib.MXFP4 if case["format"] == "mx" else lib.NVFP4
    q, s, t = state["A"]
    tp = t.data_ptr() if t is not None else None
    if k != "product":
        x = state["x"]
        rows, cols = x.shape
        lib.oscars_quantize_fp4(x.data_ptr(), x.stride(0), dt, rows, cols, fmt, q.data_ptr(), q.stride(0), s.data_ptr(), tp, stream=stream)
        if k == "codes":
            out = state["out"]
            lib.oscars_dequantize_fp4(q.data_ptr(), q.stride(0), s.data_ptr(), tp, fmt, rows, cols, out.data_ptr(), cols, dt, stream=stream)
            return out
    else:   # the calls take codes as bytes (what quantisation writes is bytes already)
        if "bytes" not in state:   # a buffer of the program's, written in each pass
            state["bytes"] = torch.empty(q.shape, device=DEV, dtype=torch.uint8)
        q = state["bytes"].copy_(q)
    M, N, K = case["M"], case["N"], case["K"]
    qb, sb, tb = state["B"]
    if "weight" not in state:   # laid out once, as a program keeps its weights
        state["weight"] = qb.to(torch.uint8)
    qb = state["weight"]
    C = state["C"]
    lib.oscars_gemm_fp4_nt(q.data_ptr(), q.stride(0), s.data_ptr(), qb.data_ptr(), qb.stride(0), sb.data_ptr(), fmt, C.data_ptr(), N, dt,
                           M, N, K, row_scale_a_ptr=tp, row_scale_b_ptr=tb.data_ptr() if tb is not None else None,
                           bias_ptr=state["bias"].data_ptr() if case["bias"] else None, relu=case["relu"], stream=stream)
    return C


# ------------------------------------------------------------------ 64 bits
def _round32(v):
    """fp64 rounded to fp32's values (every definition's intermediate result is kept in 32 bits)."""
    return v.to(torch.float32).to(torch.float64)


def _exact_codes(x, fmt):
    """(values in 4 bits with their block scales, row scales or None) in 64 bits, by arithmetic: a value is rounded to
    a multiple of the step of its binade."""
    rows, cols = x.shape
    n = BLOCK[fmt]
    blocks = (cols + n - 1) // n
    X = torch.zeros(rows, blocks * n, dtype=torch.float64, device=DEV)
    X[:, :cols] = x.to(torch.float64)
    X = X.view(rows, blocks, n)
    m = X.abs().max(dim=2).values
    t = None
    if fmt == "mx":
        p = torch.floor(torch.log2(torch.where(m > 0, m, torch.ones_like(m))))
        p = torch.where(torch.exp2(p) > m, p - 1, torch.where(torch.exp2(p + 1) <= m, p + 1, p))
        scale = torch.exp2(torch.where(m > 0, torch.clamp(p - 2, min=-127.0), torch.full_like(p, -127.0)))
        u = X.abs() / scale.unsqueeze(2)
    else:
        top = m.max(dim=1).values
        t = torch.where(top > 0, torch.clamp(_round32(top / 2688.0), min=2.0 ** -110), torch.zeros_like(top))
        safe = torch.where(t > 0, t, torch.ones_like(t))
        want = torch.clamp(_round32(m * _round32(1.0 / _round32(6.0 * safe)).unsqueeze(1)), max=448.0)
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(want, min=2.0 ** -20))), min=-6.0) - 3.0)
        scale = torch.round(want / step) * step
        s = _round32(scale * t.unsqueeze(1))
        r = torch.where(s > 0, _round32(1.0 / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(s))
        u = _round32(X.abs() * r.unsqueeze(2))
    step = torch.where(u < 2.0, 0.5, torch.where(u < 4.0, 1.0, 2.0)).to(torch.float64)
    v = torch.clamp(torch.round(u / step) * step, max=6.0) * torch.sign(X) * scale.unsqueeze(2)
    return v.view(rows, -1)[:, :cols], t


def _exact_kept(kept, rows, cols, fmt):
    """The values that packed codes and tiled scales stand for, in 64 bits, by the bits' meaning."""
    q, s, t = kept
    n = BLOCK[fmt]
    r = torch.arange(rows, device=DEV).unsqueeze(1)
    c = torch.arange(cols, device=DEV).unsqueeze(0)
    per = ((cols + n - 1) // n + 3) // 4
    j = c // n
    byte = s[(r // 128 * per + j // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + j % 4].to(torch.int64)
    code = (q[:, torch.arange(cols, device=DEV) // 2].to(torch.int64) >> (4 * (c % 2))) & 15
    e, f = (code >> 1) & 3, (code & 1).to(torch.float64)
    v = torch.where(e == 0, 0.5 * f, torch.exp2((e - 1).to(torch.float64)) * (1.0 + 0.5 * f))
    v = torch.where(code >= 8, -v, v)
    if fmt == "mx":
        return v * torch.exp2((byte - 127).to(torch.float64)), None
    e, f = (byte >> 3) & 15, (byte & 7).to(torch.float64) / 8.0
    return v * torch.where(e == 0, f * 2.0 ** -6, (1.0 + f) * torch.exp2((e - 7).to(torch.float64))), t.to(torch.float64)


def exact(case, seed):
    """The definitions in 64 bits: the norm by sums over the last axis, codes by arithmetic, products term by term."""
    st = prepare(case, seed)
    k = case["kind"]
    if k in ("norm", "grad"):
        n, r, c = case["groups"], case["rows"], case["cols"]
        out, stats, sums = [], [], []
        for i in range(n):   # one group after the other
            x = st["x"][i * r:(i + 1) * r].to(torch.float64)
            gamma, beta = st["gamma"][i].to(torch.float64), st["beta"][i].to(torch.float64)
            if k == "norm":
                mean = torch.sum(x, 1) / c
                var = torch.sum(torch.square(x - mean.unsqueeze(1)), 1) / c
                rstd = torch.rsqrt(var + EPS)
                out.append(torch.addcmul(beta, (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), gamma))
                stats.append((mean, rstd))
                continue
            dy = st["dy"][i * r:(i + 1) * r].to(torch.float64)
            mean, rstd = st["mean"][i * r:(i + 1) * r].to(torch.float64), st["rstd"][i * r:(i + 1) * r].to(torch.float64)
            xh = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
            u = torch.mv(dy, gamma) / c
            v = torch.mv(dy * xh, gamma) / c
            out.append((dy * gamma - u.unsqueeze(1) - xh * v.unsqueeze(1)) * rstd.unsqueeze(1))
            sums.append((torch.einsum("rc,rc->c", dy, xh), torch.einsum("rc->c", dy)))
        if k == "norm":
            return {"y": torch.cat(out), "mean": torch.cat([m for m, _ in stats]), "rstd": torch.cat([s for _, s in stats])}
        return {"dx": torch.cat(out), "dgamma": torch.stack([a for a, _ in sums]), "dbeta": torch.stack([b for _, b in sums])}
    fmt = case["format"]
    if k == "codes":
        v, t = _exact_codes(st["x"], fmt)
        return v if t is None else v * t.unsqueeze(1)
    M, N, K = case["M"], case["N"], case["K"]
    A, ta = _exact_codes(st["x"], fmt) if k == "layer" else _exact_kept(st["A"], M, K, fmt)
    B, tb = _exact_kept(st["B"], N, K, fmt)
    y = torch.empty(M, N, dtype=torch.float64, device=DEV)
    for i in range(0, M, 1024):
        y[i:i + 1024] = torch.mm(A[i:i + 1024], B.t())
    if fmt == "nv":
        y *= torch.outer(ta, tb)
    if case["bias"]:
        y += st["bias"].to(torch.float64)
    return y.clamp_(min=0.0) if case["relu"] else y
