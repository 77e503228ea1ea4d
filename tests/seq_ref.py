"""Float64 references of the token-sequence operators and the bounds their tests use.

U = 2^-24 is the relative error of one fp32 rounding (24 significant bits), UB = 2^-8 that of one to
bf16 (8 bits): half a step each.  Bounds are worst cases over every order of the operations, worked
out element by element beside the reference value itself.
"""

from __future__ import annotations

import torch

F64 = torch.float64
U, UB = 2.0 ** -24, 2.0 ** -8
TINY = 2.0 ** -120   # what fp32 and bf16 may flush to zero, and the sums of it


def io_dtype(io):
    return torch.bfloat16 if io == "bf16" else torch.float32


def stored(ref, err, io):
    """The bound after the result, within ``err`` of ``ref``, is rounded to its storage."""
    return err + (UB if io == "bf16" else U) * (ref.abs() + err) + TINY


def assert_within(got, ref, bound, what):
    """Elementwise; non-finite values of the reference have to be met exactly."""
    got = got.detach().to(F64).cpu()
    ref, bound = ref.cpu(), bound.cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    finite = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), f"{what}: infinities differ"
    assert bool(torch.isfinite(got[finite]).all()), f"{what}: not finite"
    over = (got[finite] - ref[finite]).abs() - bound[finite]
    if over.numel() and float(over.max()) > 0:
        i = int(over.argmax())
        raise AssertionError(f"{what}: {float(got[finite][i])} against {float(ref[finite][i])}, "
                             f"bound {float(bound[finite][i])}")


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------
def embed_backward(ids, grad_out, V, scale, io):
    """(grad_table, bound): a row's count of additions, and the scaling."""
    ids, g = ids.cpu().long(), grad_out.cpu().to(F64)
    at = torch.nonzero((ids >= 0) & (ids < V))[:, 0]
    ref = torch.zeros((V, g.shape[1]), dtype=F64).index_add_(0, ids[at], g[at])
    mag = torch.zeros((V, g.shape[1]), dtype=F64).index_add_(0, ids[at], g[at].abs())
    count = torch.bincount(ids[at], minlength=V)[:V].to(F64)[:, None]
    ref, mag = scale * ref, abs(scale) * mag
    return ref, stored(ref, (count + 1) * 1.01 * U * mag, io)


# ---------------------------------------------------------------------------
# Gated scan
# ---------------------------------------------------------------------------
def scan(x, g, gate, leaky, io, h0=None, lengths=None, grad_h=None, grad_last=None):
    """Step by step in float64 with every output's bound: {name: (value, bound)}.

    The decay's relative error is (|g| + 6) U: |g| U from rounding the exponential's
    argument, its own last place, the sum 1 + e and the reciprocal.  Any order of products and
    sums gives a term at most two more roundings a step that it lives through, so a term that
    is s steps old is off by at most s (|g| + 8) U of itself."""
    x, g = x.cpu().to(F64), g.cpu().to(F64)
    T, b, D = x.shape
    if gate == "sigmoid":
        a, na, ea = torch.sigmoid(g), torch.sigmoid(-g), (g.abs().clamp(max=200.0) + 6) * U
    else:
        a, na, ea = g, 1 - g, torch.zeros_like(g)
    w = na if leaky else torch.ones_like(na)
    # 1 - g of a decay given as it is is one rounding off
    ew = (ea if gate == "sigmoid" else torch.full_like(g, U)) if leaky else torch.zeros_like(g)
    length = torch.full((b,), T) if lengths is None else lengths.cpu().long().clamp(0, T)
    h = torch.zeros((b, D), dtype=F64) if h0 is None else h0.cpu().to(F64)
    S, E = h.abs(), torch.zeros((b, D), dtype=F64)   # sum of the terms' sizes, error
    before, ebefore, sbefore = [], [], []
    hs, eh = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(T):
        on = (t < length)[:, None]
        before.append(h), ebefore.append(E), sbefore.append(S)
        aa = a[t].abs()
        term = w[t].abs() * x[t].abs()
        h = torch.where(on, a[t] * h + w[t] * x[t], h)
        E = torch.where(on, aa * (E + (ea[t] + 3 * U) * S) + (ew[t] + 3 * U) * term, E)
        S = torch.where(on, aa * S + term, S)
        hs[t], eh[t] = torch.where(on, h, 0.0), torch.where(on, E, 0.0)
    out = dict(h=(hs, stored(hs, eh, io)), h_last=(h, stored(h, E, "f32")))
    if grad_h is None:
        return out
    dh = grad_h.cpu().to(F64)
    c = torch.zeros((b, D), dtype=F64) if grad_last is None else grad_last.cpu().to(F64)
    Sc, Ec = c.abs(), torch.zeros((b, D), dtype=F64)
    gx, gg, ex, eg = (torch.zeros_like(x) for _ in range(4))
    for t in range(T - 1, -1, -1):
        on = (t < length)[:, None]
        lam, Sl = dh[t] + c, dh[t].abs() + Sc
        El = Ec + 2 * U * Sl
        wx, aa = w[t].abs(), a[t].abs()
        gx[t] = torch.where(on, w[t] * lam, 0.0)
        ex[t] = torch.where(on, wx * (El + (ew[t] + U) * Sl), 0.0)
        d = before[t] - x[t] if leaky else before[t]
        sd = sbefore[t] + x[t].abs() if leaky else sbefore[t]
        ed = ebefore[t] + 2 * U * sd
        f = a[t] * na[t] if gate == "sigmoid" else torch.ones_like(lam)
        ef = 2 * ea[t] + 4 * U
        gg[t] = torch.where(on, lam * d * f, 0.0)
        eg[t] = torch.where(on, f.abs() * (El * sd + Sl * ed + ef * Sl * sd), 0.0)
        Ec = torch.where(on, aa * (El + (ea[t] + 3 * U) * Sl), Ec)
        Sc = torch.where(on, aa * Sl, Sc)
        c = torch.where(on, a[t] * lam, c)
    out.update(grad_x=(gx, stored(gx, ex, io)), grad_g=(gg, stored(gg, eg, io)), grad_h0=(c, stored(c, Ec, "f32")))
    return out


def scan_loss(x, g, gate, leaky, h0, lengths, grad_h, grad_last):
    """sum(grad_h * h) + sum(grad_last * h_last) in float64 (a smooth function of x, g, h0)."""
    T = x.shape[0]
    a = torch.sigmoid(g) if gate == "sigmoid" else g
    w = (1 - a) if leaky else torch.ones_like(a)
    h, total = h0, 0.0
    for t in range(T):
        on = torch.ones_like(h, dtype=torch.bool) if lengths is None else (t < lengths)[:, None].expand_as(h)
        h = torch.where(on, a[t] * h + w[t] * x[t], h)
        total = total + (torch.where(on, h, 0.0) * grad_h[t]).sum()
    return float(total + (h * grad_last).sum())


# ---------------------------------------------------------------------------
# Linear cross entropy
# ---------------------------------------------------------------------------
def ce(hidden, weight, targets, scale, io, row_weight=None, train=True):
    """{name: (value, bound)} in float64, where the inputs are (a GPU's float64 products).

    A logit is off by at most (D + 2) U of the sum of its products' sizes.  dz of the loss is
    off by that twice (the logit and lse), by the exponentials' own error, (|z - lse| + 8) U,
    and in bf16 by its rounding; products of V (or N) terms add that many U of their terms."""
    dev = weight.device
    h, w = hidden.to(F64), weight.to(F64)
    N, D = h.shape
    V = w.shape[0]
    t = targets.to(dev).long()
    keep = (t >= 0) & (t < V)
    h = torch.where(keep[:, None], h, 0.0)
    at = t.clamp(0, V - 1)
    r = torch.ones((N,), dtype=F64, device=dev) if row_weight is None else row_weight.to(F64)
    r = torch.where(keep, r, 0.0) * scale
    z = scale * torch.matmul(h, w.t())
    ez = (D + 2) * U * abs(scale) * torch.matmul(h.abs(), w.abs().t())
    lse = torch.logsumexp(z, dim=1)
    # the statistics: every term's error, and V additions at worst (tile by tile)
    p = torch.exp(z - lse[:, None])
    live = torch.isfinite(z)
    top = torch.where(live, ez, 0.0).max(dim=1).values
    away = torch.where(live, (z - lse[:, None]).abs(), 0.0)
    el = top + (p * (away + 8) * U).sum(dim=1) + (V / 64 + 80) * U + 2 * U * lse.abs()
    chosen = z.gather(1, at[:, None])[:, 0]
    echo = ez.gather(1, at[:, None])[:, 0]
    loss = lse - chosen
    out = dict(loss=(torch.where(keep, loss, 0.0),
                     torch.where(keep, stored(loss, el + echo + U * (lse.abs() + chosen.abs()), "f32"), 0.0)),
               lse=(torch.where(keep, lse, 0.0), torch.where(keep, stored(lse, el, "f32"), 0.0)))
    if not train:
        return out
    onehot = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    dz = r[:, None] * (p - onehot)
    ep = r[:, None].abs() * (p * (ez + el[:, None] + (away + 8) * U) + 3 * U * (p + onehot))
    rounding = UB if io == "bf16" else 2 * U
    edz = ep + rounding * dz.abs()
    gh, gw = torch.matmul(dz, w), torch.matmul(dz.t(), h)
    # (the sums over classes and rows run in pieces whose sums are added: their length bounds both)
    egh = torch.matmul(edz + (V + 8) * U * dz.abs(), w.abs())
    egw = torch.matmul((edz + (N + 8) * U * dz.abs()).t(), h.abs())
    gh = torch.where(keep[:, None], gh, 0.0)
    egh = torch.where(keep[:, None], egh, 0.0)
    out.update(grad_hidden=(gh, stored(gh, egh, io)), grad_weight=(gw, stored(gw, egw, io)))
    # independent roundings of dz (and of the stored result) add up in the mean square: the
    # 2-norm's bound is the root of the summed squares, one half step each at most
    out["norms"] = dict(
        grad_hidden=rounding * float((torch.matmul(dz.square(), w.square()).sum() + gh.square().sum()).sqrt()),
        grad_weight=rounding * float((torch.matmul(dz.square().t(), h.square()).sum() + gw.square().sum()).sqrt()))
    return out


def ce_loss(hidden, weight, targets, scale, row_weight):
    """sum(row_weight * loss) over the rows that have a target, in float64."""
    keep = (targets >= 0) & (targets < weight.shape[0])
    z = scale * torch.matmul(hidden[keep], weight.t())
    loss = torch.logsumexp(z, dim=1) - z.gather(1, targets[keep].long()[:, None])[:, 0]
    return float((row_weight[keep] * loss).sum())
