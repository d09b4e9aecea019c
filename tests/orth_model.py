"""The orthogonalisation with the roundings that its header states, in 64-bit
arithmetic on one matrix: the operands X, S and b S + c S^2 of the products in
half at the kernels' powers of two; X itself, the diagonal of S and, in the
last two steps, that of b S + c S^2 in float32 (in the others what its
rounding leaves is)."""
import torch


def _half(x, scale):
    return (x * scale).half().double() / scale


def _single(x):
    return x.float().double()


def model(G, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, scale_x=256.0, diagonals_apart=True):
    """scale_x: X's power of two, 2^8 (2^5 on the path of one launch).
    `diagonals_apart` false: S and P rounded whole."""
    a, b, c = coefficients
    X = G.double()
    tall = X.shape[0] > X.shape[1]
    X = X.t() if tall else X
    X = _single(X / (X.square().sum().sqrt() + eps))
    for step in range(steps):
        x = _half(X, scale_x)
        S = x @ x.t()
        if not diagonals_apart:
            S = _half(S, 1024.0)
            X = _single(a * X + _half(b * S + c * (S @ S), 256.0) @ x)
            continue
        d = _single(torch.diag(S))
        So = _half(S - torch.diag(torch.diag(S)), 1024.0)
        S2 = So @ So
        P = (b + c * (d[:, None] + d)) * So + c * S2
        p = _single((b + c * d) * d + c * torch.diag(S2))
        kept = 0 * p if step + 2 >= steps else _half(p, 256.0)
        P = _half(P - torch.diag(torch.diag(P)), 256.0) + torch.diag(kept)
        X = _single((a + p - kept)[:, None] * X + P @ x)
    return X.t() if tall else X


def bound(want, exact):
    """How far a result that has the model's roundings may lie from the model
    `want`: the actual rounding r of the model to bfloat16, and as much as all
    its roundings together cost, d = |want - exact|, since a 32-bit sum next to
    a rounding's tie decides it the other way: the two are independent,
    sqrt(r^2 + d^2), and their product averages out over the elements (2 %)."""
    r = (want.bfloat16().double() - want).norm()
    d = (want - exact).norm()
    return 1.02 * (r * r + d * d).sqrt()
