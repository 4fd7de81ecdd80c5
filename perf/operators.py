"""Timed cases of the server's orthogonalised update and of the 8-bit products
that a trained model answers with.

* ``orth``: updates of ``batch`` weight matrices are orthogonalised by
  Newton-Schulz steps (``oscars_orthogonalize``): X = G / (|G| + eps), then
  ``steps`` times A = X X^T, X <- a X + (b A + c A^2) X; the result is scale X;
* ``merge``: the server merges pushed deltas of one weight matrix into its
  momentum, orthogonalises it and applies it to the global model in one call
  (``oscars_merge_orthogonal``);
* ``product``: an 8-bit product with a scale for each token (row of A) and each
  channel (row of B), bias and ReLU in its epilogue (``oscars_gemm_i8_nt``), its
  operands already in 8 bits;
* ``layer``: a dense layer of a model kept in 8 bits: tokens in bf16 or fp32
  are quantised row by row (``oscars_quantize_i8``) and multiplied.

Where ``own`` is false, ``run`` computes the same in elementary torch
operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
COEFF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the smallest matrix of a server step: the 10-class head of the 784-512-10 model
        {"name": "orth-10x512-f32", "kind": "orth", "batch": 1, "rows": 10, "cols": 512, "dtype": "f32", "steps": 5, "pad": 0},
        # sixteen workers' updates of that model's hidden layer in one call
        {"name": "orth-16x512x784-bf16", "kind": "orth", "batch": 16, "rows": 512, "cols": 784, "dtype": "bf16", "steps": 5, "pad": 0},
        # a tall ragged matrix whose rows are further apart than its width
        {"name": "orth-1001x333-f32", "kind": "orth", "batch": 3, "rows": 1001, "cols": 333, "dtype": "f32", "steps": 5, "pad": 6},
        # the square hidden layer of the three-layer workload, fp32 throughout
        {"name": "orth-1024x1024-f32", "kind": "orth", "batch": 1, "rows": 1024, "cols": 1024, "dtype": "f32", "steps": 5, "pad": 0},
        # a wide projection of a large model
        {"name": "orth-4096x4096-bf16", "kind": "orth", "batch": 1, "rows": 4096, "cols": 4096, "dtype": "bf16", "steps": 5, "pad": 0},
        # a round's server step on the headline model's hidden layer: 16 pushed deltas, momentum
        {"name": "merge-512x784-w16", "kind": "merge", "rows": 512, "cols": 784, "workers": 16, "steps": 5, "nesterov": True, "shift": 0},
        # the same away from round sizes: odd rows and columns, buffers that start between 16-byte boundaries
        {"name": "merge-1537x385-w3", "kind": "merge", "rows": 1537, "cols": 385, "workers": 3, "steps": 5, "nesterov": False, "shift": 1},
        # a single sample through the headline model's hidden layer: latency alone
        {"name": "layer-1x512x784-bf16", "kind": "layer", "M": 1, "N": 512, "K": 784, "dtype": "bf16", "bias": True, "relu": True},
        # sixteen samples through a large projection: the weights' bytes are what counts
        {"name": "layer-16x4096x4096-bf16", "kind": "layer", "M": 16, "N": 4096, "K": 4096, "dtype": "bf16", "bias": False, "relu": False},
        # the held-out set of the headline model through its hidden layer
        {"name": "layer-8192x512x784-f32", "kind": "layer", "M": 8192, "N": 512, "K": 784, "dtype": "f32", "bias": True, "relu": True},
        # ragged operands already in 8 bits, fp32 out
        {"name": "product-777x1003x1537-f32", "kind": "product", "M": 777, "N": 1003, "K": 1537, "dtype": "f32", "bias": True, "relu": False},
        # a long prompt or a large evaluation batch through a large projection
        {"name": "product-8192x4096x4096-bf16", "kind": "product", "M": 8192, "N": 4096, "K": 4096, "dtype": "bf16", "bias": False, "relu": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """One more case of the same ranges, no more work than the largest listed one."""
    largest = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= largest:
            return case


def _draw(rng):
    kind = rng.choice(["orth", "orth", "merge", "product", "layer"])
    if kind == "orth":
        return {"kind": kind, "batch": rng.choice([1, 1, 1, _log_int(rng, 1, 32)]), "rows": _log_int(rng, 1, 4096),
                "cols": _log_int(rng, 1, 4096), "dtype": rng.choice(["f32", "bf16"]), "steps": rng.choice([5, 5, 5, 3, 8]),
                "pad": rng.choice([0, 0, 0, 1, 24])}
    if kind == "merge":
        return {"kind": kind, "rows": _log_int(rng, 1, 2048), "cols": _log_int(rng, 1, 2048), "workers": _log_int(rng, 1, 32),
                "steps": 5, "nesterov": rng.random() < 0.5, "shift": rng.choice([0, 0, 1, 2, 3])}
    return {"kind": kind, "M": _log_int(rng, 1, 8192), "N": _log_int(rng, 1, 8192), "K": _log_int(rng, 1, 8192),
            "dtype": rng.choice(["f32", "bf16"]), "bias": rng.random() < 0.5, "relu": rng.random() < 0.5}


def work(case):
    k = case["kind"]
    if k in ("orth", "merge"):
        # the products of a step, the two symmetric ones counted for one triangle
        r, c = case["rows"], case["cols"]
        s, ln, batch = min(r, c), max(r, c), case.get("batch", 1)
        flops = batch * case["steps"] * (s * (s + 1) * ln + s * s * (s + 1) + 2 * s * s * ln)
        if k == "orth":
            return {"bytes": batch * r * c * 2 * (4 if case["dtype"] == "f32" else 2), "flops": flops}
        # deltas in, model and momentum in and out
        return {"bytes": 4 * r * c * (case["workers"] + 4), "flops": flops + 2 * r * c * (case["workers"] + 2)}
    M, N, K = case["M"], case["N"], case["K"]
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": M * K * (size if k == "layer" else 1) + N * K + 4 * N + (4 * N if case["bias"] else 0)
            + (0 if k == "layer" else 4 * M) + M * N * size, "flops": 2 * M * N * K}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _update(g, rows, cols, noise):
    """What an accumulated mini-batch gradient looks like: a sum of outer
    products of output gradients and activations, decaying, and noise."""
    r = min(64, rows, cols)
    d = torch.randn(rows, r, device=DEV, generator=g) * torch.linspace(1.0, 0.1, r, device=DEV)
    x = torch.randn(r, cols, device=DEV, generator=g)
    return 1e-3 * ((d @ x) / math.sqrt(r) + noise * torch.randn(rows, cols, device=DEV, generator=g))


def prepare(case, seed):
    g = _gen(seed)
    k = case["kind"]
    if k == "orth":
        b, r, c, ld = case["batch"], case["rows"], case["cols"], case["cols"] + case["pad"]
        G = torch.zeros(b, r, ld, device=DEV, dtype=_dtype(case))
        for i in range(b):
            G[i, :, :c] = _update(g, r, c, 0.3).to(G.dtype)
        return {"case": case, "G": G, "O": torch.empty(b, r, c, device=DEV, dtype=G.dtype)}
    if k == "merge":
        r, c, sh = case["rows"], case["cols"], case["shift"]

        def shifted(t):
            buf = torch.empty(r * c + sh, device=DEV)
            buf[sh:] = t.reshape(-1)
            return buf[sh:]

        common = _update(g, r, c, 0.1)
        deltas = [shifted(common + _update(g, r, c, 0.3)) for _ in range(case["workers"])]
        lim = 1.0 / math.sqrt(c)
        x = shifted((torch.rand(r, c, device=DEV, generator=g) * 2 - 1) * lim)
        v = shifted(_update(g, r, c, 0.3))
        return {"case": case, "x": x, "v": v, "deltas": deltas, "w": [1.0 / case["workers"]] * case["workers"]}
    M, N, K = case["M"], case["N"], case["K"]
    ld = (K + 15) // 16 * 16

    def in_8_bits(x):   # the checkpoint's weights, or tokens that the layer before left in 8 bits
        s = x.abs().amax(1) / 127.0
        q = torch.zeros(x.shape[0], ld, device=DEV, dtype=torch.int8)
        q[:, :K] = torch.round(x / s[:, None]).to(torch.int8)
        return q, s

    W = torch.randn(N, K, device=DEV, generator=g) / math.sqrt(K)
    st = {"case": case, "C": torch.empty(M, N, device=DEV, dtype=_dtype(case)),
          "bias": torch.randn(N, device=DEV, generator=g) * 0.1 if case["bias"] else None}
    st["B"], st["sb"] = in_8_bits(W)
    del W
    # activations: Gaussian with a few wide channels, tokens of different sizes
    x = torch.randn(M, K, device=DEV, generator=g) * torch.exp(0.5 * torch.randn(M, 1, device=DEV, generator=g))
    x *= 1.0 + 4.0 * (torch.rand(K, device=DEV, generator=g) < 0.02)
    if k == "layer":
        st["x"] = x.to(_dtype(case))
        st["A"], st["sa"] = torch.zeros(M, ld, device=DEV, dtype=torch.int8), torch.empty(M, device=DEV)
    else:
        st["A"], st["sa"] = in_8_bits(x)
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _newton_schulz(G, steps):
    tall = G.shape[-2] > G.shape[-1]
    X = G.mT if tall else G
    norm = (X.double() * X.double()).sum((-2, -1), keepdim=True).sqrt()
    X = (X / (norm + EPS)).float()
    a, b, c = COEFF
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


def _run_plain(state):
    case = state["case"]
    k = case["kind"]
    if k == "orth":
        G = state["G"][:, :, :case["cols"]].float()
        return _newton_schulz(G, case["steps"]).to(state["G"].dtype).contiguous()
    if k == "merge":
        x, v = state["x"], state["v"]
        d = torch.stack(state["deltas"]).T @ torch.tensor(state["w"], device=DEV)
        v.mul_(0.95).add_(d)
        u = d + 0.95 * v if case["nesterov"] else v
        O = _newton_schulz(u.reshape(case["rows"], case["cols"]), case["steps"])
        x.add_(O.reshape(-1), alpha=0.02)
        return {"x": x, "v": v}
    if k == "layer":
        x = state["x"].float()
        mx = x.abs().amax(1)
        sa = mx / torch.full_like(mx, 127.0)   # by a number torch would multiply with its reciprocal, a step off at times
        A = torch.round(x / sa[:, None])
    else:
        sa, A = state["sa"], state["A"][:, :case["K"]].float()
    y = (A @ state["B"][:, :case["K"]].float().T) * sa[:, None] * state["sb"]
    if case["bias"]:
        y = y + state["bias"]
    if case["relu"]:
        y = torch.relu(y)
    return y.to(state["C"].dtype)


def _run_own(state):
    import paper_2102_08550_gb300 as lib

    case = state["case"]
    k = case["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    if k in ("orth", "merge"):
        r, c, b = case["rows"], case["cols"], case.get("batch", 1)
        dt = lib.BF16 if case.get("dtype") == "bf16" else lib.F32
        if "ws" not in state:   # kept by the program, as its buffers are
            n = (lib.oscars_orthogonalize_workspace(b, r, c, dt) if k == "orth"
                 else lib.oscars_merge_orthogonal_workspace(r, c))
            state["ws"] = torch.empty(n, device=DEV, dtype=torch.uint8)
        ws = state["ws"]
        if k == "orth":
            G, O = state["G"], state["O"]
            lib.oscars_orthogonalize(G.data_ptr(), G.stride(1), G.stride(0), O.data_ptr(), O.stride(1), O.stride(0), b, r, c,
                                     dt, case["steps"], ws.data_ptr(), ws.numel(), coeff=COEFF, eps=EPS, stream=stream)
            return O
        lib.oscars_merge_orthogonal(state["x"].data_ptr(), [d.data_ptr() for d in state["deltas"]], state["w"], r, c,
                                    state["v"].data_ptr(), 0.95, case["nesterov"], 0.02, case["steps"], ws.data_ptr(),
                                    ws.numel(), coeff=COEFF, eps=EPS, stream=stream)
        return {"x": state["x"], "v": state["v"]}
    M, N, K = case["M"], case["N"], case["K"]
    A, B, C = state["A"], state["B"], state["C"]
    dt = lib.BF16 if case["dtype"] == "bf16" else lib.F32
    if k == "layer":
        x = state["x"]
        lib.oscars_quantize_i8(x.data_ptr(), x.stride(0), dt, M, K, A.data_ptr(), A.stride(0), state["sa"].data_ptr(),
                               stream=stream)
    lib.oscars_gemm_i8_nt(A.data_ptr(), A.stride(0), state["sa"].data_ptr(), B.data_ptr(), B.stride(0),
                          state["sb"].data_ptr(), C.data_ptr(), C.stride(0), dt, M, N, K,
                          bias_ptr=state["bias"].data_ptr() if case["bias"] else None, relu=case["relu"], stream=stream)
    return C


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The definition in 64 bits: the polynomial applied from the other side
    (columns' Gram matrix where `run` takes the rows'), the sums term by term."""
    st = prepare(case, seed)
    k = case["kind"]
    if k in ("orth", "merge"):
        r, c = case["rows"], case["cols"]
        if min(r, c) ** 2 * max(r, c) * case.get("batch", 1) * case["steps"] > 4096 ** 3 * 6:
            return None
        v = None
        if k == "orth":
            X = st["G"][:, :, :c].to(torch.float64)
        else:
            d = sum(wk * dk.to(torch.float64) for wk, dk in zip(st["w"], st["deltas"]))
            v = 0.95 * st["v"].to(torch.float64) + d
            X = ((d + 0.95 * v) if case["nesterov"] else v).reshape(1, r, c)
        X = X / (torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True) + EPS)
        flip = r > c
        if flip:
            X = X.transpose(1, 2).contiguous()
        eye = torch.eye(X.shape[1], dtype=torch.float64, device=DEV)
        a, b, cc = COEFF
        for _ in range(case["steps"]):
            S = torch.einsum("bik,bjk->bij", X, X)
            X = torch.einsum("bij,bjk->bik", a * eye + torch.einsum("bij,bjk->bik", S, b * eye + cc * S), X)
        if flip:
            X = X.transpose(1, 2)
        if k == "orth":
            return X.contiguous()
        return {"x": st["x"].to(torch.float64) + 0.02 * X.reshape(-1), "v": v}
    M, N, K = case["M"], case["N"], case["K"]
    if k == "layer":
        # the scale is kept in 32 bits, and a code is the nearest integer (ties to
        # even) of the quotient in 32 bits: both are the operator's definition
        x = st["x"].to(torch.float64)
        sa = (x.abs().max(dim=1).values / 127.0).to(torch.float32).to(torch.float64)
        A = torch.round((x / sa.unsqueeze(1)).to(torch.float32)).to(torch.float64)
    else:
        sa, A = st["sa"].to(torch.float64), st["A"][:, :K].to(torch.float64)
    y = torch.empty(M, N, dtype=torch.float64, device=DEV)
    Bt = (st["B"][:, :K].to(torch.float64) * st["sb"].to(torch.float64).unsqueeze(1)).t()
    for i in range(0, M, 1024):
        y[i:i + 1024] = torch.mm(A[i:i + 1024], Bt) * sa[i:i + 1024].unsqueeze(1)
    if case["bias"]:
        y += st["bias"].to(torch.float64)
    return y.clamp_(min=0.0) if case["relu"] else y
