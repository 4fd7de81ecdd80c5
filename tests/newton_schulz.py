"""Newton-Schulz steps in 64 bits, and how far the roundings of an implementation
may move them: every stored value is perturbed by its rounding's size and every
product by its accumulation's, and the divergence is measured (test
infrastructure; runs where its tensors are)."""
import torch

MUON = (3.4445, -4.7750, 2.0315)
# bounds of one rounding, relative to the value: X and the factors of an fp32
# result are kept as two fp16 halves (11 + 11 bits, the second half rounded: 2^-22);
# a bf16 result rounds A and the factor to fp16 (2^-11)
STORE = 2.0 ** -22
FACTOR = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -11}
# accumulation: the tensor core cuts up to 2^-23 of the running sum at each addition
# of 16 products, four to twelve of them (64 of K, one to three products) before the
# sum moves to fp32 registers, or K / 16 for bf16 results, whose factors are coarser
ACC = 2.0 ** -21


def _rel(x, size, g):
    return x if g is None else x * (1 + size * (2 * torch.rand(x.shape, generator=g, dtype=x.dtype, device=x.device) - 1))


def newton_schulz(G, steps, coeff=MUON, eps=1e-7, gen=None, dtype=torch.float32):
    """O of one matrix in 64 bits; with `gen`, one perturbed run."""
    a, b, c = (torch.tensor(v, dtype=torch.float32).double().item() for v in coeff)   # the call takes fp32 ones
    X = G.double()
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    X = X / (X.square().sum().sqrt() + torch.tensor(eps, dtype=torch.float32).double().item())
    X = _rel(X, STORE, gen)
    eye = torch.eye(X.shape[0], dtype=torch.float64, device=X.device)

    def product(P, Q):
        R = P @ Q
        if gen is not None:   # accumulation: relative to the norms of the row and the column
            size = P.norm(dim=1, keepdim=True) * Q.norm(dim=0, keepdim=True)
            R = R + ACC * size * (2 * torch.rand(R.shape, generator=gen, dtype=R.dtype, device=R.device) - 1)
        return R

    f = FACTOR[dtype]
    for k in range(steps):
        A = product(_rel(X, f, gen), _rel(X, f, gen).T)
        if gen is not None and c != 0:   # as it is computed: c (A + b / 2c)^2 + (a - b^2 / 4c), A + b / 2c stored
            A = _rel(A + b / (2 * c) * eye, f, gen)
            B = _rel((a - b * b / (4 * c)) * eye + c * product(A, A), f, gen)
        else:
            B = _rel(a * eye + b * A + c * product(A, A), f, gen)
        X = _rel(product(B, _rel(X, f, gen) if k + 1 == steps else X), STORE, gen)   # the last step's X as the factors
    return X.T if tall else X


def envelope(G, steps, dtype, coeff=MUON, eps=1e-7):
    """(reference, Frobenius and largest divergence of two perturbed runs, each relative)."""
    ref = newton_schulz(G, steps, coeff, eps)
    fro = big = 0.0
    for seed in (11, 12):
        gen = torch.Generator(device=G.device).manual_seed(seed)
        d = newton_schulz(G, steps, coeff, eps, gen, dtype) - ref
        fro = max(fro, (d.norm() / ref.norm()).item())
        big = max(big, (d.abs().max() / ref.abs().max()).item())
    return ref, fro, big
