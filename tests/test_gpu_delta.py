"""Gated delta rule on the GPU against the recurrence in float64."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import block_ref, seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


def make(cfg, seed, ragged=False, carry=False, layout="time", decay=0.3):
    gen = torch.Generator().manual_seed(seed)
    dt, T, b, H, Hk = seq_ref.io_dtype(cfg.io), cfg.T, cfg.batch, cfg.H, cfg.Hk or cfg.H
    n = lambda *s: torch.randn(s, generator=gen)
    lead = (b, T) if layout == "batch" else (T, b)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    rows = [unit(n(*lead, Hk, cfg.K)).flatten(-2), unit(n(*lead, Hk, cfg.K)).flatten(-2), n(*lead, H * cfg.V)]
    if layout == "fused":
        both = torch.cat(rows, -1).to(dt)
        rows = list(both.split([x.shape[-1] for x in rows], -1))
    q, k, v = (x.to(dt).unflatten(-1, (h, -1)) for x, h in zip(rows, (Hk, Hk, H)))
    g = (-decay * torch.rand((*lead, H), generator=gen)).to(dt)
    beta = torch.sigmoid(n(*lead, H)).to(dt)
    go = n(*lead, H, cfg.V).to(dt)
    if layout == "batch":
        q, k, v, g, beta, go = (x.transpose(0, 1) for x in (q, k, v, g, beta, go))
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (b,), generator=gen, dtype=torch.int32)
        lengths[0] = 0
        lengths[-1] = T + 7   # clamped
    state = (b, H, cfg.K, cfg.V)
    return dict(q=q, k=k, v=v, g=g, beta=beta, grad_o=go, lengths=lengths, s0=0.3 * n(*state) if carry else None,
                grad_last=n(*state) if carry else None)


def run(cfg, d, dev):
    m = {k: None if v is None else v.to(dev) for k, v in d.items()}
    seen = [m[k] for k in ("q", "k", "v", "g", "beta")]
    o, last, ckpt = dendsn.delta_rule(cfg, *seen, m["s0"], m["lengths"])
    out = dict(o=o, s_last=last)
    out.update(dendsn.delta_rule_backward(cfg, *seen, m["lengths"], ckpt, m["grad_o"], m["grad_last"]))
    return out


def same_bits(a, b, what):
    assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), what


def check(cfg, d, dev):
    got = run(cfg, d, dev)
    scale = cfg.K ** -0.5 if cfg.scale is None else cfg.scale
    for k, (value, bound) in block_ref.delta(d, scale, cfg.io).items():
        seq_ref.assert_within(got[k], value, bound, k)
    again = run(cfg, d, dev)
    for k in got:
        same_bits(got[k], again[k], k)
    return got


# steps around a chunk's 64 and its tiles of 16; head sizes around a fragment's 8, a step's 32,
# a tile's 16 and the widths of 64 and 128
SHAPES = [(1, 1, 1, 0, 1, 1), (1, 2, 3, 0, 16, 8), (2, 1, 2, 1, 64, 33), (15, 1, 1, 0, 8, 16), (16, 2, 2, 0, 32, 32),
          (17, 1, 4, 2, 33, 31), (63, 1, 2, 0, 65, 40), (64, 2, 1, 0, 128, 64), (65, 1, 3, 1, 100, 7), (96, 1, 2, 0, 7, 130),
          (128, 1, 1, 0, 64, 32), (130, 3, 6, 2, 60, 100), (200, 1, 2, 0, 127, 65), (257, 1, 1, 0, 24, 200)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,b,H,Hk,K,V", SHAPES)
def test_against_recurrence(gpu_device, T, b, H, Hk, K, V, io):
    for ragged, carry, layout in ((False, False, "time"), (True, True, "fused"), (False, True, "batch")):
        cfg = dendsn.DeltaRuleConfig(T=T, batch=b, H=H, Hk=Hk, K=K, V=V, io=io)
        announce(f"delta {cfg} ragged {ragged} carry {carry} {layout}")
        check(cfg, make(cfg, T + K, ragged, carry, layout), gpu_device)


# few heads and so many steps that they are cut into segments; ends inside, at and between them
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,b,H,Hk,K,V", [(1100, 1, 1, 0, 16, 20), (1537, 3, 2, 1, 36, 33), (700, 4, 1, 0, 128, 17)])
def test_segments(gpu_device, T, b, H, Hk, K, V, io):
    for ragged, carry, layout in ((False, True, "time"), (True, True, "fused"), (False, False, "batch")):
        cfg = dendsn.DeltaRuleConfig(T=T, batch=b, H=H, Hk=Hk, K=K, V=V, io=io)
        announce(f"delta segments {cfg} ragged {ragged} carry {carry} {layout}")
        d = make(cfg, T + K, ragged, carry, layout, decay=0.02)
        if ragged and b > 2:
            d["lengths"][1] = 256
        check(cfg, d, gpu_device)


# so many heads that a block takes 32 columns of v; of both widths, of K that is a multiple of 8 and not
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("K", [16, 21, 72, 69])
def test_many_heads(gpu_device, K, io):
    cfg = dendsn.DeltaRuleConfig(T=70, batch=8, H=32, Hk=16, K=K, V=32 if K != 21 else 31, io=io)
    announce(f"delta many heads {cfg}")
    check(cfg, make(cfg, K, True, True, "fused"), gpu_device)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_scale_and_decays(gpu_device, io):
    """Decays of 1, decays that forget all (minus infinity among them), betas of 0 and 1, a scale."""
    cfg = dendsn.DeltaRuleConfig(T=100, batch=2, H=2, K=32, V=32, io=io, scale=-1.5)
    d = make(cfg, 3, carry=True)
    d["g"][:, 0] = 0.0
    d["g"][40:44, 1, 0] = -float("inf")
    d["g"][70, 1, 1] = -1000.0
    d["beta"][10:20] = 0.0
    d["beta"][20:30] = 1.0
    announce(f"delta decays {io}")
    got = run(cfg, d, gpu_device)
    ref = block_ref.delta(dict(d, g=d["g"].clamp_min(-200.0)), cfg.scale, io)
    for k, (value, bound) in ref.items():
        seq_ref.assert_within(got[k], value, bound, k)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_equal_keys(gpu_device, io):
    """All keys alike and betas of 1: every step replaces what the one before wrote."""
    cfg = dendsn.DeltaRuleConfig(T=80, batch=1, H=1, K=16, V=16, io=io)
    d = make(cfg, 5)
    d["k"] = torch.zeros_like(d["k"])
    d["k"][..., 3] = 1.0
    d["beta"] = torch.ones_like(d["beta"])
    announce(f"delta equal keys {io}")
    check(cfg, d, gpu_device)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_past_the_end(gpu_device, io):
    """What inputs hold past a sequence's end (NaN, infinities) reaches nothing; outputs are +0 there."""
    cfg = dendsn.DeltaRuleConfig(T=90, batch=3, H=2, Hk=1, K=20, V=24, io=io)
    d = make(cfg, 7, carry=True)
    d["lengths"] = torch.tensor([70, 0, 90], dtype=torch.int32)
    announce(f"delta past the end {io}")
    clean = run(cfg, d, gpu_device)
    for i, name in enumerate(("q", "k", "v", "g", "beta", "grad_o")):
        d[name] = d[name].clone()
        d[name][70:, 0] = float("nan") if i % 2 else float("inf")
        d[name][:, 1] = float("nan")
    got = run(cfg, d, gpu_device)
    for k in got:
        same_bits(got[k], clean[k], k)
    for k in ("o", "grad_q", "grad_k", "grad_v", "grad_g", "grad_beta"):
        for x in (got[k][70:, 0], got[k][:, 1]):
            assert not x.contiguous().view(torch.uint8).any(), k
    same_bits(got["s_last"][1].cpu(), d["s0"][1], "the state of a sequence of no steps")
    same_bits(got["grad_s0"][1].cpu(), d["grad_last"][1], "its gradient")


def test_broadcast_inputs(gpu_device):
    """Gates and queries that are one row for all steps: strides of 0."""
    cfg = dendsn.DeltaRuleConfig(T=70, batch=2, H=2, K=16, V=16)
    d = make(cfg, 9)
    for n in ("g", "beta", "q"):
        d[n] = d[n][:1].expand(cfg.T, *d[n].shape[1:])
    announce("delta broadcast")
    dev = gpu_device
    m = {k: None if v is None else v.to(dev) for k, v in d.items()}
    for n in ("g", "beta", "q"):
        m[n] = m[n][:1].expand(cfg.T, *m[n].shape[1:])
        assert m[n].stride(0) == 0
    o, last, ckpt = dendsn.delta_rule(cfg, *(m[k] for k in ("q", "k", "v", "g", "beta")))
    ref = block_ref.delta(d, cfg.K ** -0.5, "f32")
    seq_ref.assert_within(o, *ref["o"], "o")
    back = dendsn.delta_rule_backward(cfg, *(m[k] for k in ("q", "k", "v", "g", "beta")), None, ckpt, m["grad_o"])
    for k, x in back.items():
        seq_ref.assert_within(x, *ref[k], k)


def test_gradients_against_differences(gpu_device):
    """The loss's change along a direction, from the recurrence at two points: central differences
    of step e in float64 are off by e^2 of the third derivative."""
    cfg = dendsn.DeltaRuleConfig(T=70, batch=1, H=2, Hk=1, K=12, V=10)
    d = make(cfg, 11, carry=True)
    announce("delta differences")
    got = run(cfg, d, gpu_device)
    gen = torch.Generator().manual_seed(12)
    names = ("q", "k", "v", "g", "beta", "s0")
    way = {n: torch.randn(d[n].shape, generator=gen, dtype=torch.float64) for n in names}

    def loss(e):
        x = {n: d[n].double() + e * way[n] for n in names}
        ref = block_ref.delta(dict(d, **x), cfg.K ** -0.5, "f32", train=False)
        return (ref["o"][0] * d["grad_o"].double()).sum() + (ref["s_last"][0] * d["grad_last"].double()).sum()

    for n in names:
        full, way = way, {m: w if m == n else torch.zeros_like(w) for m, w in way.items()}
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        way = full
        mine = (got["grad_" + n].double().cpu() * way[n]).sum()
        size = (got["grad_" + n].double().cpu().norm() * way[n].norm())
        assert abs(slope - mine) <= 1e-5 * size, (n, slope, mine)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("b,H,Hk,K,V", [(1, 1, 0, 1, 1), (3, 4, 2, 64, 64), (5, 3, 1, 33, 31), (2, 2, 0, 128, 130), (4, 2, 0, 100, 36)])
def test_step(gpu_device, b, H, Hk, K, V, io):
    """One token on slots against the recurrence: a product and a sum a value and step, sums of K."""
    cfg = dendsn.DeltaRuleConfig(T=1, batch=b, H=H, Hk=Hk, K=K, V=V, io=io)
    d = make(cfg, b + K, carry=True)
    gen = torch.Generator().manual_seed(2)
    held = torch.randn((b + 3, H, K, V), generator=gen)
    slots = torch.randperm(b + 3, generator=gen)[:b].to(torch.int32)
    if b > 2:
        slots[1], slots[2] = -1, b + 3
    on = (slots >= 0) & (slots < b + 3)
    d["s0"] = held[slots.clamp(0, b + 2).long()]
    announce(f"delta step {cfg}")
    ref = block_ref.delta(dict(d, grad_last=None), K ** -0.5, io, train=False)
    state = held.to(gpu_device)
    seen = [d[k][0].to(gpu_device) for k in ("q", "k", "v", "g", "beta")]
    o = dendsn.delta_rule_step(cfg, *seen, state, slots.to(gpu_device)).cpu()
    want, bound = ref["o"]
    seq_ref.assert_within(o[on], want[0][on], bound[0][on], "o")
    assert not o[~on].float().any()
    seq_ref.assert_within(state.cpu()[slots[on].long()], ref["s_last"][0][on], ref["s_last"][1][on], "state")
    rest = torch.ones(b + 3, dtype=torch.bool)
    rest[slots[on].long()] = False
    same_bits(state.cpu()[rest], held[rest], "states that no request names")


def test_steps_continue_a_prompt(gpu_device):
    """A prompt in one call, then token by token on its last state: as the whole in one call."""
    cfg = dendsn.DeltaRuleConfig(T=140, batch=2, H=2, K=32, V=48, io="bf16")
    d = make(cfg, 21)
    announce("delta prompt and steps")
    m = [d[k].to(gpu_device) for k in ("q", "k", "v", "g", "beta")]
    o, last, _ = dendsn.delta_rule(cfg, *m, save_ckpt=False)
    head = cfg.with_(T=100)
    _, state, _ = dendsn.delta_rule(head, *(x[:100] for x in m), save_ckpt=False)
    outs = [dendsn.delta_rule_step(cfg.with_(T=1), *(x[t] for x in m), state) for t in range(100, 140)]
    ref = block_ref.delta(d, 32 ** -0.5, "bf16", train=False)
    seq_ref.assert_within(torch.stack(outs), ref["o"][0][100:], ref["o"][1][100:], "o")
    seq_ref.assert_within(state, *ref["s_last"], "state")
    seq_ref.assert_within(last, *ref["s_last"], "s_last")


def test_empty(gpu_device):
    z = lambda *s: torch.zeros(s, device=gpu_device)
    cfg = dendsn.DeltaRuleConfig(T=0, batch=2, H=3, K=4, V=5)
    s0 = torch.randn((2, 3, 4, 5), device=gpu_device)
    o, last, ckpt = dendsn.delta_rule(cfg, z(0, 2, 3, 4), z(0, 2, 3, 4), z(0, 2, 3, 5), z(0, 2, 3), z(0, 2, 3), s0)
    assert o.shape == (0, 2, 3, 5) and torch.equal(last, s0)
    back = dendsn.delta_rule_backward(cfg, z(0, 2, 3, 4), z(0, 2, 3, 4), z(0, 2, 3, 5), z(0, 2, 3), z(0, 2, 3), None, ckpt,
                                      z(0, 2, 3, 5), s0)
    assert torch.equal(back["grad_s0"], s0)
    none = cfg.with_(T=4, batch=0)
    o, last, _ = dendsn.delta_rule(none, z(4, 0, 3, 4), z(4, 0, 3, 4), z(4, 0, 3, 5), z(4, 0, 3), z(4, 0, 3))
    assert o.numel() == 0 and last.numel() == 0
