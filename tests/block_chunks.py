"""The gated delta rule and its gradients over chunks of 64 steps, in float64 on the CPU, and what the
kernels' results may be off by in norm.

The formulas are those of the head of csrc/seq/seq_delta.hip; that they are the recurrence's is a test of
its own.  ``planes``: values that are computed on the way are rounded to fp32 and taken as a sum of that
many bf16 values wherever they are operands of a product, as the scans do.  ``leave_out``: names of
terms of the decay's gradient ("after", "before", "held") that are left out: mistakes, planted here.

How far off, in norm over the steps and values of one head of one sequence (U, UB, UP: one rounding to
fp32, to bf16, to a pair of bf16 values).  Errors that fall either way add in squares.

States (s_last, grad_s0) hang on operands of three bf16 values, which hold all of fp32, so only fp32's own
roundings count.  In a chunk there are as many in a row as a value has matrix instructions, which round
their running sum: of a sum over K 3 K / 32 (fp32: K / 4), of T's product 2 x 6 (16), of the state's 2 x 3
(16); four of R and the decays; and 16 + 3 x 16 of T.  A chunk's errors decay with the state that they
are in; where the states' memory is long (half of a chunk's state is left after the next) their squares
add to twice one chunk's at most.  Segments go through all that twice and through a join of K / 4:

    off <= sqrt(2 n) U,   n = (3 K / 32 + 12 + 6 | K / 4 + 32) + 68,   segments: 2 n + K / 4.

Other results pass six such sums, in bf16 with operands of two values (UP):

    off <= 6 (sqrt(2 n) U + [bf16] UP), twice that for gradients, and the rounding to io.

The gradient of the logarithmic decay adds up to 64 terms q.dq and k.dk, each a sum over K whose errors
fall either way: sqrt(64 / K) of what dq and dk are off by times |q| and |k|, in norm over the steps.
"""

from __future__ import annotations

import torch

from tests.block_ref import UP
from tests.seq_ref import F64, TINY, U, UB

CHUNK = 64
TERMS = ("after", "before", "held")


def split(x, planes):
    if not planes:
        return x
    left, out = x.to(torch.float32), torch.zeros_like(x)
    for _ in range(planes):
        part = left.to(torch.bfloat16).to(torch.float32)
        out += part.to(F64)
        left = left - part
    return out


def sequence(q, k, v, g, beta, s0, grad_o, grad_last, scale, planes=0, leave_out=()):
    """One sequence of n steps: q, k [H, n, K] (a head each), v, grad_o [H, n, V], g, beta [H, n], s0,
    grad_last [H, K, V]."""
    n, S, kept = q.shape[1], s0, []
    o, r = [], lambda x: split(x, planes)
    lower = torch.ones((CHUNK, CHUNK), dtype=torch.bool).tril()
    t_ = lambda x: x.transpose(-1, -2)
    for c in range(0, n, CHUNK):
        q1, k1, v1, g1, b1 = (x[:, c:c + CHUNK] for x in (q, k, v, g, beta))
        m = q1.shape[1]
        G = torch.cumsum(g1, 1)
        D = torch.exp((G[:, :, None] - G[:, None, :]).masked_fill(~lower[:m, :m], -float("inf")))
        A = (b1[..., None] * D * (k1 @ t_(k1))).tril(-1)
        T = r(torch.linalg.solve_triangular(torch.eye(m, dtype=F64) + A, torch.eye(m, dtype=F64).expand_as(A), upper=False))
        P = r(scale * D * (q1 @ t_(k1)))
        eg, tail, whole = torch.exp(G)[..., None], torch.exp(G[:, -1:] - G)[..., None], torch.exp(G[:, -1])[:, None, None]
        R = b1[..., None] * (v1 - eg * (k1 @ r(S)))
        U_ = T @ r(R)
        o.append(scale * eg * (q1 @ r(S)) + P @ r(U_))
        kept.append((q1, k1, v1, b1[..., None], D, T, P, eg, tail, whole, S, U_))
        S = whole * S + t_(k1) @ r(tail * U_)
        if planes:
            S = S.to(torch.float32).to(F64)
    out = dict(o=torch.cat(o, 1) if o else torch.zeros_like(v), s_last=S)
    if grad_o is None:
        return out
    dS, parts = grad_last, []
    for i in reversed(range(len(kept))):
        q1, k1, v1, b1, D, T, P, eg, tail, whole, S, U_ = kept[i]
        do = grad_o[:, i * CHUNK:(i + 1) * CHUNK]
        dU = t_(P) @ do + tail * (k1 @ r(dS))
        dR = t_(T) @ r(dU)
        E = scale * D * (do @ t_(U_))
        diag = torch.diagonal(E, dim1=-2, dim2=-1)[..., None]
        E = E.tril(-1)
        F = (-D * (dR @ t_(U_))).tril(-1)
        dq = scale * eg * (do @ t_(S)) + E @ k1
        X = F @ k1 - eg * (dR @ t_(S))
        Y1, Y2 = tail * (U_ @ t_(dS)), t_(E) @ q1 + t_(b1 * F) @ k1
        kx = (k1 * X).sum(-1)
        after = (q1 * dq).sum(-1) + b1[..., 0] * kx - (k1 * Y2).sum(-1)
        before = (k1 * Y1).sum(-1)
        held = (whole * S * dS).sum((-1, -2))[:, None]
        dg = {"after": after.flip(1).cumsum(1).flip(1), "before": before.cumsum(1) - before, "held": held.expand_as(after)}
        dq, dk = dq + diag * k1, b1 * X + Y1 + Y2 + diag * q1
        parts.append((dq, dk, b1 * dR, sum(x for name, x in dg.items() if name not in leave_out), (dR * v1).sum(-1) + kx,
                      q1.norm(dim=-1) * dq.norm(dim=-1) + k1.norm(dim=-1) * dk.norm(dim=-1)))
        dS = whole * dS + t_(q1) @ r(scale * eg * do) - t_(k1) @ r(b1 * eg * dR)
        if planes:
            dS = dS.to(torch.float32).to(F64)
    names = ("grad_q", "grad_k", "grad_v", "grad_g", "grad_beta", "terms")
    for name, x in zip(names, zip(*reversed(parts))):
        out[name] = torch.cat(x, 1)
    out["grad_s0"] = dS
    return out


def delta(d, scale, **kw):
    """As ``sequence`` for inputs ``d`` of the calls' layout [T, batch, heads, *], whatever lengths: a dict
    of outputs [T, batch, heads, *] (states [batch, H, K, V]), and ``terms`` [T, batch, H]."""
    T, b, Hk, K = d["q"].shape
    H, V = d["v"].shape[2:]
    wide = {n: d[n].to(F64).cpu() for n in ("q", "k", "v", "g", "beta", "grad_o")}
    for n in "qk":
        wide[n] = wide[n].repeat_interleave(H // Hk, 2)
    state = lambda x: torch.zeros((b, H, K, V), dtype=F64) if x is None else x.to(F64).cpu()
    s0, last = state(d["s0"]), state(d["grad_last"])
    res = dict(o=torch.zeros((T, b, H, V), dtype=F64), s_last=s0.clone(), grad_s0=last.clone())
    res.update(grad_q=torch.zeros((T, b, H, K), dtype=F64), grad_k=torch.zeros((T, b, H, K), dtype=F64),
               grad_v=torch.zeros((T, b, H, V), dtype=F64))
    res.update({n: torch.zeros((T, b, H), dtype=F64) for n in ("grad_g", "grad_beta", "terms")})
    for i in range(b):
        n = T if d["lengths"] is None else max(0, min(T, int(d["lengths"][i])))
        if n == 0:
            continue
        x = {name: t[:n, i].transpose(0, 1) for name, t in wide.items()}
        one = sequence(x["q"], x["k"], x["v"], x["g"], x["beta"], s0[i], x["grad_o"], last[i], scale, **kw)
        for name, t in one.items():
            if name in ("s_last", "grad_s0"):
                res[name][i] = t
            else:
                res[name][:n, i] = t.transpose(0, 1)
    for name in ("grad_q", "grad_k"):
        res[name] = res[name].unflatten(2, (Hk, H // Hk)).sum(3)
    return res


def over_head(name, x):
    """Norms [batch, heads] of an output."""
    if name in ("s_last", "grad_s0"):
        return x.to(F64).cpu().flatten(2).norm(dim=-1)
    x = x.to(F64).cpu()
    return (x if x.dim() == 4 else x[..., None]).transpose(0, 1).transpose(1, 2).flatten(2).norm(dim=-1)


def bounds(ref, K, io, segments=False):
    """What each output may be off by in norm, [batch, heads] each."""
    n = (3 * K / 32 + 18 if io == "bf16" else K / 4 + 32) + 68
    state = (2 * (2 * n + K / 4 if segments else n)) ** 0.5 * U
    one = 6 * (state + (UP if io == "bf16" else 0.0))
    kept = UB if io == "bf16" else U
    out = {}
    for name, x in ref.items():
        size = over_head(name, x)
        if name in ("s_last", "grad_s0"):
            out[name] = state * size
        elif name == "grad_g":
            out[name] = kept * size + 2 * one * (64 / K) ** 0.5 * over_head(name, ref["terms"])
        elif name != "terms":
            out[name] = (kept + (one if name == "o" else 2 * one)) * size
    return {name: x + TINY for name, x in out.items()}


def off(got, ref, name):
    return over_head(name, got.to(F64).cpu() - ref[name])
