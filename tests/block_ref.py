"""Float64 references of a block's operators, and what their tests allow.

The delta rule's references are the recurrence itself, step by step, differentiated by torch.

What the kernels may be off by (U = 2^-24 and UB = 2^-8 are the relative errors of one rounding
to fp32 and bf16; a pair of bf16 values is off by UP = 2^-17 at most: 2^-8 of the half step that
the first leaves).  Of a chunk every result is a sum of at most n = K + 64 products of values
that went through at most six such sums before (decays, T, R, U, the state, P or E); one sum in
fp32 is off by at most n U of its terms' magnitudes, each operand by U or UP.  Keys are of unit
length, betas below 1, decays at most 1: a step multiplies what the state is off by with
a matrix of norm 1 at most, so chunks add theirs.  With signs that fall either way the terms'
root mean square counts, not their sum, and n becomes its root:

    off <= 6 (sqrt(n) U + [bf16] UP) chunks, of the result's root mean square over the tensor,

for a value at eight such deviations (no test has more than 2^20 values: a normal deviate of
8 has a chance of 2^-50).  The gradients pass the chunk's sums twice.  The logarithmic decay's
gradient is a sum over up to 64 steps of differences of terms q_i.dq_i and k_i.dk_i: 8 times what one
term is off by.  A term may be far larger than the difference: with equal keys and betas of 1 each step
overwrites the one before, no decay has any effect, and terms of order 1 add up to a gradient of exactly
0, which each off by U or UP of itself leave at that times 1.  So there the size that counts is
that of |q_i| |dq_i| + |k_i| |dk_i|, which bounds a term, where it is more than the gradient's own.
"""

from __future__ import annotations

import torch

from tests.seq_ref import F64, TINY, U, UB

UP = 2.0 ** -17
TOP = 448.0


def rounded(io):
    return UB if io == "bf16" else U


def clean_norm(x):
    return x.to(F64).cpu().nan_to_num(0.0, 0.0, 0.0).norm(dim=-1)


def delta(d, scale, io, train=True):
    """References of every output of the delta rule for inputs ``d`` (q, k, v, g, beta, s0, lengths,
    grad_o, grad_last): dict of (value, bound)."""
    q, k, v, g, beta = (d[n].to(F64).cpu().requires_grad_(train) for n in ("q", "k", "v", "g", "beta"))
    T, b, Hk, K = q.shape
    H, V = v.shape[2:]
    s0 = (torch.zeros((b, H, K, V), dtype=F64) if d["s0"] is None else d["s0"].to(F64).cpu()).requires_grad_(train)
    length = torch.full((b,), T) if d["lengths"] is None else d["lengths"].cpu().long().clamp(0, T)
    S, o = s0, []
    for t in range(T):
        on = (t < length)[:, None, None]
        clean = lambda x: torch.where(on if x.dim() == 3 else on[..., 0], x, 0.0)
        qt, kt = (clean(x[t]).repeat_interleave(H // Hk, 1) for x in (q, k))
        a = torch.exp(clean(g[t]))[..., None, None]
        miss = clean(v[t]) - (kt[..., None] * (a * S)).sum(-2)
        S = torch.where(on[..., None], a * S + kt[..., None] * (clean(beta[t])[..., None] * miss)[..., None, :], S)
        o.append(torch.where(on, scale * (qt[..., None] * S).sum(-2), 0.0))
    o = torch.stack(o) if T else v.detach()
    out = dict(o=o.detach(), s_last=S.detach())
    if train:
        seed = (o * d["grad_o"].to(F64).cpu()).sum()
        if d["grad_last"] is not None:
            seed = seed + (S * d["grad_last"].to(F64).cpu()).sum()
        grads = torch.autograd.grad(seed, [q, k, v, g, beta, s0], allow_unused=True)
        for n, x, of in zip(("q", "k", "v", "g", "beta", "s0"), grads, (q, k, v, g, beta, s0)):
            out["grad_" + n] = torch.zeros_like(of) if x is None else x.detach()
    n, chunks = K + 64, max(1, -(-T // 64))
    off = 8 * 6 * (n ** 0.5 * U + (UP if io == "bf16" else 0.0)) * chunks
    times = dict(o=1, s_last=1, grad_g=16)
    kept = rounded(io)
    res = {}
    for name, x in out.items():
        rms = x[torch.isfinite(x)].square().mean().sqrt() if x.numel() else torch.zeros((), dtype=F64)
        if name == "grad_g":
            rms = torch.maximum(rms, (clean_norm(d["q"]) * out["grad_q"].norm(dim=-1) + clean_norm(d["k"]) * out["grad_k"].norm(dim=-1)
                                      ).square().mean().sqrt())
        res[name] = (x, times.get(name, 2) * off * (rms + x.abs()) + (U if name in ("s_last", "grad_s0") else kept) * x.abs() + TINY)
    return res


def norm(x, weight, residual, eps, io, grad_y=None, grad_sum=None, summed=None):
    """(value, bound) of the norm's outputs.  A row's sum of D squares is off by (D + 1) U at most,
    its root by half of that and three roundings; y by two more."""
    x, D = x.to(F64).cpu(), x.shape[1]
    s = x if residual is None else x + residual.to(F64).cpu()
    one = rounded(io)
    power = s.square().mean(1, keepdim=True) + eps
    rstd = power ** -0.5
    w = torch.ones((D,), dtype=F64) if weight is None else weight.to(F64).cpu()
    rel = (0.5 * (D + 6) + 4) * U  # of rstd, where s is exact to U
    y = s * rstd * w
    out = dict(rstd=(rstd[:, 0], rel * rstd[:, 0]), y=(y, (rel + 4 * U + one) * y.abs() + TINY))
    if residual is not None:
        out["sum"] = (s, (one + U) * s.abs() + TINY)
    if grad_y is not None:
        # the backward reads the rounded sum: what it is given is what counts
        if summed is not None:
            s = summed.to(F64).cpu()
        gy = grad_y.to(F64).cpu()
        hat, gw = s * rstd, gy * w
        along = (gw * hat).mean(1, keepdim=True)
        gx = rstd * (gw - hat * along)
        mean_off = (rel + (D + 8) * U) * (gw * hat).abs().mean(1, keepdim=True)
        off = rstd * ((rel + 6 * U) * gw.abs() + hat.abs() * (mean_off + (2 * rel + 6 * U) * along.abs()))
        if grad_sum is not None:
            gx = gx + grad_sum.to(F64).cpu()
        out["grad_x"] = (gx, off + (one + U) * (gx.abs() + off) + TINY)
        terms = gy * hat
        gwt = terms.sum(0)
        off = (rel + (x.shape[0] + 4) * U) * terms.abs().sum(0)
        out["grad_weight"] = (gwt, off + one * (gwt.abs() + off) + TINY)
    return out


def adamw(p, g, m, v, step, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.01, scale=1.0):
    """(value, bound) of a step from fp32 arrays: m and v after two products and a sum, and the
    constants' own rounding (4 U); the update after a root, a quotient and four roundings more."""
    p, g, m, v = (x.to(F64).cpu() for x in (p, g, m, v))
    g = g * scale
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    off_m = 5 * U * ((b1 * m).abs() + ((1 - b1) * g).abs()) + TINY
    off_v = 6 * U * v1 + TINY
    f1, f2 = 1 - b1 ** step, 1 - b2 ** step
    root = (v1 / f2).sqrt() + eps
    to = m1 / f1 / root
    off_to = off_m / f1 / root + to.abs() * 14 * U + TINY
    p1 = p - lr * (wd * p + to)
    off_p = lr * (off_to + 4 * U * ((wd * p).abs() + to.abs())) + 2 * U * (p.abs() + p1.abs())
    return dict(p=(p1, off_p), m=(m1, off_m), v=(v1, off_v))


def e4m3_spacing(x):
    """The distance of the two e4m3 values around |x| (of which the lower may be x)."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6)))) / 8
