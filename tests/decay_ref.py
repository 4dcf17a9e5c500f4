"""Plain 64-bit forms of attention with a decaying bias, for the tests.

Each returns, beside its result, the sum of the magnitudes of the terms that the
result adds up: an operand that is off by a part delta moves the result by at most
delta times that sum, whatever cancels in it.
"""
import math

import torch

F64 = torch.float64

# What every weight, state and product may be off by, as a part of itself.
#
# fp32 results: the exponent of phi, |W x| + ||x||^2 / 2 <= 40 at the tests' sizes, carries the
# roundings of its product, its constant and their sum, at most 3 x 40 x 2^-24 = 7e-6 of phi for q
# and as much for k; sums of up to 256 terms in a register and between chunks add
# 2^-24 sqrt(256) and less: 4e-5 covers twice the total.
# bf16 results: phi(q) and phi(k) are operands of one term, off by 2^-8 of themselves at most; the
# exponents carry W's two terms, 2^-17 |W| |x| <= 22 x 2^-17 for q and for k, and P and the state two
# terms, 2^-16 each: 2 x 2^-8 + 4.5e-4 with what fp32 results have, below 2.2 x 2^-8.
# Gradients of bf16 rows: all that is computed (phi(q), phi(k), the state, G, R, W) has two terms:
# 6 x 2^-16 + 3.4e-4 + 4e-5 = 4.7e-4, below 2^-11; twice that for the two sums that dq and dk go through.
DELTA = {torch.float32: 4e-5, torch.bfloat16: 2.2 * 2.0 ** -8}
GRAD_DELTA = {torch.float32: 4e-5, torch.bfloat16: 2.0 ** -10}
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step of the result's own type
STATE_DELTA = 4e-5  # states are fp32 results in either case


def phi(x, W, nprf=False, features="prf"):
    """phi of x [..., rows, d], W [m, d], and the rows it was taken of (normalised with nprf)."""
    x = x.to(F64)
    if nprf:
        norm = x.norm(dim=-1, keepdim=True)
        x = torch.where(norm > 0, x / norm, torch.zeros_like(x))
    if features == "elu":
        return torch.where(x > 0, x + 1, x.clamp(max=0).exp()), x
    W = W.to(F64)
    return (x @ W.T - 0.5 * (x * x).sum(-1, keepdim=True)).exp() / math.sqrt(W.shape[0]), x


def _ones(v):
    return torch.cat([v, torch.ones_like(v[..., :1])], dim=-1)


def weights(n, rate, device):
    """e^{-rate (i - j)} for j <= i, zero after (a rate of inf: the diagonal)."""
    at = torch.arange(n, device=device, dtype=F64)
    dist = at[:, None] - at
    w = torch.where(dist > 0, (-rate * dist.clamp(min=1)).exp(), (dist == 0).to(F64))
    return w


def _power(rate, steps):
    return float(math.exp(-rate * steps)) if steps else 1.0


def prompt(q, k, v, rate, W, state=None, nprf=False, features="prf"):
    """One sequence and head: z [n, d], its scale, the state behind it and its scale."""
    n = q.shape[0]
    fq, fk = phi(q, W, nprf, features)[0], phi(k, W, nprf, features)[0]
    vh = _ones(v.to(F64))
    A = (fq @ fk.T) * weights(n, rate, q.device)
    num, mag = A @ vh, A @ vh.abs()
    left = torch.tensor([_power(rate, n - 1 - j) for j in range(n)], dtype=F64, device=q.device)[:, None]
    last, lmag = (vh * left).T @ fk, (vh.abs() * left).T @ fk
    if state is not None:
        s = state.to(F64)
        since = torch.tensor([_power(rate, i + 1) for i in range(n)], dtype=F64, device=q.device)[:, None]
        num, mag = num + since * (fq @ s.T), mag + since * (fq @ s.abs().T)
        last, lmag = last + _power(rate, n) * s, lmag + _power(rate, n) * s.abs()
    z = num[:, :-1] / num[:, -1:]
    return z, mag[:, :-1] / num[:, -1:] + z.abs(), last, lmag


def gradients(q, k, v, rate, W, dz, nprf=False, features="prf"):
    """One sequence and head: {name: (gradient, scale)} of sum(dz z) for q, k and v."""
    n = q.shape[0]
    (fq, uq), (fk, uk) = phi(q, W, nprf, features), phi(k, W, nprf, features)
    v, dz = v.to(F64), dz.to(F64)
    C = weights(n, rate, q.device)
    A = (fq @ fk.T) * C
    den = A.sum(-1, keepdim=True)
    z = A @ v / den
    g = dz / den
    gd = -(g * z).sum(-1, keepdim=True)
    gdm = (g.abs() * (A @ v.abs() / den)).sum(-1, keepdim=True)
    R, Rm = (g @ v.T + gd) * C, (g.abs() @ v.abs().T + gdm) * C
    out = {"dv": (A.T @ g, A.T @ g.abs())}
    for name, x, u, f, df, dfm in (("dq", q, uq, fq, R @ fk, Rm @ fk), ("dk", k, uk, fk, R.T @ fq, Rm.T @ fq)):
        if features == "elu":
            slope = torch.where(u > 0, torch.ones_like(u), u.clamp(max=0).exp())
            dx, mag = df * slope, dfm * slope
        else:
            W64 = W.to(F64)
            dx = (df * f) @ W64 - u * (df * f).sum(-1, keepdim=True)
            mag = (dfm * f) @ W64.abs() + u.abs() * (dfm * f).sum(-1, keepdim=True)
        if nprf:
            norm = x.to(F64).norm(dim=-1, keepdim=True)
            inv = torch.where(norm > 0, 1 / norm, torch.zeros_like(norm))
            dx = (dx - u * (u * dx).sum(-1, keepdim=True)) * inv
            mag = (mag + u.abs() * (u.abs() * mag).sum(-1, keepdim=True)) * inv
        out[name] = (dx, mag)
    return out


def tree(q, k, v, parent, rate, W, state=None, nprf=False, features="prf"):
    """z [T, d] of one tree and head and its scale (zeros where a node has no valid parents)."""
    T = q.shape[0]
    fq, fk = phi(q, W, nprf, features)[0], phi(k, W, nprf, features)[0]
    vh = _ones(v.to(F64))
    s = torch.zeros((vh.shape[1], fq.shape[1]), dtype=F64, device=q.device) if state is None else state.to(F64)
    fade = _power(rate, 1)
    behind, z, scale = {-1: (s, s.abs())}, torch.zeros_like(v, dtype=F64), torch.zeros_like(v, dtype=F64)
    for t in range(T):
        p = int(parent[t])
        if p < -1 or p >= t or p not in behind:
            continue
        new = torch.outer(vh[t], fk[t])
        behind[t] = (fade * behind[p][0] + new, fade * behind[p][1] + new.abs())
        num, mag = behind[t][0] @ fq[t], behind[t][1] @ fq[t]
        z[t] = num[:-1] / num[-1]
        scale[t] = mag[:-1] / num[-1] + z[t].abs()
    return z, scale


def excess(got, ref, scale, dtype, delta=None):
    """The largest error in units of what is allowed: delta scale + half a step of the type."""
    got, ref = got.to(F64), ref.to(F64)
    tiny = torch.finfo(torch.float32).tiny
    allowed = (DELTA[dtype] if delta is None else delta) * scale + ROUND[dtype] * ref.abs() + tiny
    err = (got - ref).abs() / allowed
    return float(err.nan_to_num(nan=float("inf")).max()) if err.numel() else 0.0
