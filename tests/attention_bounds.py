"""Attention under any mask, and its gradients, in 64 bits, each with a bound of a kernel's error.

u: a rounding to the 16-bit type.  A score is a float32 sum of dim products: its error moves a probability by at most
    delta = 2^-20 + 2 (dim + 4) 2^-24 scale |q| |k|     relative
(the exponential, the row's statistics, the sum).  A probability is rounded once more for the product with v, and the result once:
    |out - exact| <= u |out| + (u + delta) P |v|.
S' = P (D - delta_row) is rounded once for its products; D is a float32 sum, delta_row is formed of the rounded out.  float16: probabilities are rounded to steps
of 2^-24 (the largest is 256 or less), results to steps of 2^-24 too, and S' to such steps where the largest |dO| has become 1/4 to 1/2.
bfloat16: a float32 number below 2^-126 may become zero.  So may a probability, which moves out by 2^-126 |v| and S' by 2^-126 |D - delta_row|, and so may S'
itself; and a result.
"""
import math

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def formulas(torch, q, k, v, ok, scale, dtype, dout=None):
    """q [queries, heads, dim], k, v [keys, kv_heads, dim] of one sequence, ok [queries, keys].  [(exact, bound)] of out and, with dout, of dq, dk, dv."""
    u, dim, group = UNIT[dtype], q.shape[-1], q.shape[1] // k.shape[1]
    Q, K, V = q.double().transpose(0, 1), *(t.double().transpose(0, 1).repeat_interleave(group, 0) for t in (k, v))
    S = (Q @ K.transpose(-1, -2) * scale).masked_fill(~ok, -math.inf)
    most = S.amax(-1, keepdim=True) if S.shape[-1] else torch.zeros_like(S.sum(-1, keepdim=True))
    P = torch.exp(S - torch.where(most > -math.inf, most, 0.0))
    total = P.sum(-1, keepdim=True)
    P = P / torch.where(total > 0, total, 1.0)
    delta = 2.0 ** -20 + 2 * (dim + 4) * 2.0 ** -24 * scale * (Q.abs() @ K.abs().transpose(-1, -2))
    delta = delta + (P * delta).sum(-1, keepdim=True)  # a row's statistics move with its scores
    O = P @ V
    small = torch.where(ok, 2.0 ** -24 if dtype == "f16" else 2.0 ** -126, 0.0)

    def found(exact, bound, keys=False):
        e, b = (t.unflatten(0, (-1, group)).sum(1) if keys else t for t in (exact, bound))
        return e.transpose(0, 1), (u * e.abs() + b + (2.0 ** -25 if dtype == "f16" else 2.0 ** -126)).transpose(0, 1)

    out = found(O, ((u + delta) * P + small) @ V.abs())
    if dout is None:
        return [out]
    dO = dout.double().transpose(0, 1)
    D = dO @ V.transpose(-1, -2)
    dS = P * (D - (dO * O).sum(-1, keepdim=True))
    e_row = (dO.abs() * (u * O.abs() + ((u + delta) * P + small) @ V.abs())).sum(-1, keepdim=True)
    E = (u + delta) * dS.abs() + P * ((dim + 4) * 2.0 ** -23 * (dO.abs() @ V.abs().transpose(-1, -2)) + e_row)
    if dtype == "bf16":
        E = E + 2.0 ** -126 * (1 + (D - (dO * O).sum(-1, keepdim=True)).abs())
    elif dO.numel():
        E = E + 2.0 ** -22 * dO.abs().amax()
    E = torch.where(ok, E, 0.0)
    return [out, found(dS @ K * scale, E @ K.abs() * scale),
            found(dS.transpose(-1, -2) @ Q * scale, E.transpose(-1, -2) @ Q.abs() * scale, True),
            found(P.transpose(-1, -2) @ dO, ((u + delta) * P + small).transpose(-1, -2) @ dO.abs(), True)]


def assert_within(got, wanted, label):
    for name, g, (exact, bound) in zip(("out", "dq", "dk", "dv"), got, wanted):
        assert g.shape == exact.shape, (label, name)
        off = (g.double() - exact).abs() - bound
        assert bool((off <= 0).all()), (label, name, float(off.max()), float((g.double() - exact).abs().max()))
