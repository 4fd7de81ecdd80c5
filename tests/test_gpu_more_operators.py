"""The timed cases' own calls against their 64-bit results and their plain form: what is timed is right.

Tolerances, u = 2^-24 (half a step of fp32).
  codes: a code times its block's scale is exact or one rounding, its row's scale one more; half a step of the type.
  product, layer: block sums are exact, K / 16 of them are added up, each addition off by a step 2 u of the magnitudes' sum, which
       for K products of sizes |a| |b| is at most K max|A| max|B|; three roundings of the row scales and the bias.
  norm, gradient: D = 40 + cols / 1024 additions a row's value takes at most (64 x 512 and smaller: 256 + rows for a column's),
       so a result is off by at most D u of the sizes that come together; half a step of the type.
The plain form's sums take a term through at most 333 additions, in whatever order: less than ten times the bounds above."""
import pytest
import torch

import perf.more_operators as cases

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def case(kind, fmt, dtype):
    if kind in ("norm", "grad"):
        return {"kind": kind, "groups": 3, "rows": 20, "cols": 333, "dtype": dtype, "pad": 1}
    if kind == "codes":
        return {"kind": kind, "rows": 130, "cols": 333, "format": fmt, "dtype": dtype, "pad": 1}
    return {"kind": kind, "M": 37, "N": 150, "K": 333, "format": fmt, "dtype": dtype, "bias": True, "relu": False}


CASES = [(k, f, d) for d in ("f32", "bf16") for k, f in
         [("norm", "-"), ("grad", "-")] + [(k, f) for k in ("codes", "product", "layer") for f in ("mx", "nv")]]


def sizes(c, st, want):
    """What an output's roundings are relative to, by name."""
    if c["kind"] == "codes":
        return {"": 2 * U * want[""].abs()}
    if c["kind"] in ("product", "layer"):
        K, fmt = c["K"], c["format"]
        A, ta = cases._exact_codes(st["x"], fmt) if c["kind"] == "layer" else cases._exact_kept(st["A"], c["M"], K, fmt)
        B, tb = cases._exact_kept(st["B"], c["N"], K, fmt)
        S = A.abs() @ B.abs().T
        if ta is not None:
            S = S * ta[:, None] * tb
        return {"": 2 * U * (K / 16 + 2) * S + 4 * U * (S + st["bias"].abs())}
    n, r, cols = c["groups"], c["rows"], c["cols"]
    D = 40 + cols / 1024
    x = st["x"].double()
    g = st["gamma"].double().repeat_interleave(r, 0)
    if c["kind"] == "norm":
        size, d = x.abs().mean(1), x - x.mean(1, keepdim=True)
        var = (d * d).mean(1)
        rstd = (var + cases.EPS).rsqrt()
        dm = (D + 1) * U * size
        dr = 0.5 * ((D + 4) * U * var + dm * dm) / (var + cases.EPS) + 3 * U
        return {"mean": dm, "rstd": dr * rstd,
                "y": g.abs() * rstd[:, None] * (dm[:, None] + U * d.abs()) + (g * d * rstd[:, None]).abs() * (dr[:, None] + 3 * U) + U * want["y"].abs()}
    dy, mean, rstd = st["dy"].double(), st["mean"].double()[:, None], st["rstd"].double()[:, None]
    xh, h = (x - mean) * rstd, dy * g
    T = h.abs() + 2 * h.abs().mean(1, keepdim=True) + 2 * xh.abs() * (h * xh).abs().mean(1, keepdim=True)
    return {"dx": rstd * T * (D + 8) * U, "dgamma": (260 + r) * U * (dy * xh).abs().view(n, r, cols).sum(1),
            "dbeta": (260 + r) * U * dy.abs().view(n, r, cols).sum(1)}


def named(out):
    return out if isinstance(out, dict) else {"": out}


def ran(c, seed, own):
    before, cases.own = cases.own, own
    try:
        return {k: v.clone() for k, v in named(cases.run(cases.prepare(c, seed))).items()}
    finally:
        cases.own = before


@pytest.mark.parametrize("kind,fmt,dtype", CASES)
def test_own_calls_are_right(cuda_device, kind, fmt, dtype):
    c = case(kind, fmt, dtype)
    own, plain, want = ran(c, 5, True), ran(c, 5, False), named(cases.exact(c, 5))
    tol = sizes(c, cases.prepare(c, 5), want)
    assert set(own) == set(plain) == set(want) == set(tol)
    for k, w in want.items():
        half = 0.0 if own[k].dtype == torch.float32 else torch.finfo(own[k].dtype).eps / 2
        most = (tol[k] * (1 + half) + half * w.abs()) * (1 + 2.0 ** -6) + 1e-38
        assert own[k].shape == w.shape and ((own[k].double() - w).abs() <= most).all(), k
        assert ((plain[k].double() - w).abs() <= 10 * most).all(), k


@pytest.mark.parametrize("kind,fmt", [("product", "mx"), ("product", "nv"), ("layer", "nv")])
def test_passes_of_a_state_and_of_another_are_its_own(cuda_device, kind, fmt):
    """Two states in turn, three passes: what a program keeps of its weight is that state's."""
    c = case(kind, fmt, "f32")
    want = [ran(c, s, True)[""] for s in (1, 2)]
    before, cases.own = cases.own, True
    try:
        states = [cases.prepare(c, s) for s in (1, 2)]
        for i in (0, 1, 0, 1, 1, 0):
            assert torch.equal(cases.run(states[i]), want[i])
    finally:
        cases.own = before
