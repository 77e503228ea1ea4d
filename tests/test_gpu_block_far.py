"""A block's operators on arrays whose offsets pass 32 bits: some rows checked."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import block_ref, seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


def test_norm_rows_far_apart(gpu_device):
    n, D = 300000, 8192  # 2.4e9 values, 4.9 GB an array
    gen = torch.Generator(device=gpu_device).manual_seed(1)
    x = torch.empty((n, D), dtype=torch.bfloat16, device=gpu_device)
    for i in range(0, n, 50000):
        x[i:i + 50000] = torch.randn((min(50000, n - i), D), generator=gen, device=gpu_device).to(torch.bfloat16)
    w = (1 + 0.1 * torch.randn((D,), generator=gen, device=gpu_device)).to(torch.bfloat16)
    announce("norm far")
    cfg = dendsn.RMSNormConfig(N=n, D=D, io="bf16")
    y, rstd, _ = dendsn.rms_norm(cfg, x, w)
    some = torch.tensor([0, 1, 262143, 262144, 262145, n - 1], device=gpu_device)
    back = dendsn.rms_norm_backward(cfg, x, w, rstd, x)
    ref = block_ref.norm(x[some], w, None, 1e-6, "bf16", x[some])
    seq_ref.assert_within(y[some], *ref["y"], "y")
    seq_ref.assert_within(rstd[some], *ref["rstd"], "rstd")
    seq_ref.assert_within(back["grad_x"][some], *ref["grad_x"], "grad_x")


def test_norm_more_rows_than_a_launch_has(gpu_device):
    n, D = (1 << 28) + 5, 8  # 16 rows are a block of 256 threads: 2^32 and some
    one = torch.tensor([1.0, -2.0, 0.5, 4.0, -1.0, 0.25, 3.0, -0.125], dtype=torch.bfloat16, device=gpu_device)
    x = (torch.arange(n, device=gpu_device, dtype=torch.int32) % 7 + 1).to(torch.bfloat16)[:, None] * one
    some = torch.tensor([0, 1, (1 << 27) - 1, 1 << 27, (1 << 27) + 1, (1 << 28) - 1, 1 << 28, n - 1], device=gpu_device)
    residual = one.view(1, D).expand(n, D)
    cfg = dendsn.RMSNormConfig(N=n, D=D, io="bf16")
    ref = block_ref.norm(x[some], one, residual[some], 1e-6, "bf16", x[some])
    announce("norm of many rows")
    y, rstd, total = dendsn.rms_norm(cfg, x, one, residual)
    for k, got in (("y", y), ("rstd", rstd), ("sum", total)):
        seq_ref.assert_within(got[some], *ref[k], k)
    del y
    announce("norm of many rows, e4m3")
    y8, scale, rstd8, total8 = dendsn.rms_norm_e4m3(cfg, x, one, residual)
    few = cfg.with_(N=len(some))
    want = dendsn.rms_norm_e4m3(few, x[some], one, residual[some])
    for got, w in zip((y8.view(torch.uint8), scale, rstd8, total8), (want[0].view(torch.uint8), *want[1:])):
        assert torch.equal(got[some], w)


def test_adamw_value_numbers_past_32_bits(gpu_device):
    n = (1 << 32) + 777  # 17 GB of parameters, 8-bit states
    p = torch.zeros((n,), device=gpu_device)
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device=gpu_device)
    cfg = dendsn.AdamWConfig(lr=0.125, weight_decay=0.0, state="e4m3")
    states = dendsn.adamw_states(cfg, [p])
    announce("adamw far")
    dendsn.adamw(cfg, [p], [g], states, 1, seed=1)
    m, ms, r, rs = states[0]
    ref = block_ref.adamw(torch.zeros(1), torch.full((1,), 0.5), torch.zeros(1), torch.zeros(1), 1, lr=0.125, wd=0.0)
    for at in (0, 1 << 31, (1 << 32) - 1, 1 << 32, n - 1):
        seq_ref.assert_within(p[at:at + 1], *ref["p"], f"p at {at}")
        assert float(m[at].float()) == 448.0 and float(r[at].float()) == 448.0
    assert float(p.min()) == float(p.max())
    assert float(rs[-1]) == float(rs[0]) and float(ms[-1]) == float(ms[0])


def test_delta_step_slots_far_apart(gpu_device):
    H, K, V, held = 16, 128, 128, 9000  # 2.4e9 values, 9.4 GB of states
    cfg = dendsn.DeltaRuleConfig(T=1, batch=3, H=H, K=K, V=V, io="bf16")
    gen = torch.Generator().manual_seed(2)
    n = lambda *s: torch.randn(s, generator=gen)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    d = dict(q=unit(n(1, 3, H, K)).bfloat16(), k=unit(n(1, 3, H, K)).bfloat16(), v=n(1, 3, H, V).bfloat16(),
             g=-torch.rand((1, 3, H), generator=gen).bfloat16(), beta=torch.rand((1, 3, H), generator=gen).bfloat16(),
             s0=n(3, H, K, V), lengths=None, grad_o=None, grad_last=None)
    slots = torch.tensor([8999, 0, 8192], dtype=torch.int32)
    state = torch.zeros((held, H, K, V), device=gpu_device)
    state[slots.long()] = d["s0"].to(gpu_device)
    announce("delta step far")
    o = dendsn.delta_rule_step(cfg, *(d[k][0].to(gpu_device) for k in ("q", "k", "v", "g", "beta")), state, slots.to(gpu_device))
    ref = block_ref.delta(d, K ** -0.5, "bf16", train=False)
    seq_ref.assert_within(o, ref["o"][0][0], ref["o"][1][0], "o")
    seq_ref.assert_within(state[slots.long().to(gpu_device)], *ref["s_last"], "state")
    assert not state[1:8192].any()


def test_delta_steps_far_apart(gpu_device):
    """Rows of one long tensor that lie 2^21 values apart: 64 steps span 2^28 bytes, all of them 2^32."""
    T, apart = 1100, 1 << 21
    cfg = dendsn.DeltaRuleConfig(T=T, batch=1, H=1, K=16, V=16, io="bf16")
    gen = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(s, generator=gen)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    d = dict(q=unit(n(T, 1, 1, 16)).bfloat16(), k=unit(n(T, 1, 1, 16)).bfloat16(), v=n(T, 1, 1, 16).bfloat16(),
             g=(-0.05 * torch.rand((T, 1, 1), generator=gen)).bfloat16(), beta=torch.rand((T, 1, 1), generator=gen).bfloat16(),
             s0=None, lengths=None, grad_o=n(T, 1, 1, 16).bfloat16(), grad_last=None)
    far = torch.zeros((T, apart), dtype=torch.bfloat16, device=gpu_device)
    m = {}
    for i, k in enumerate(("q", "k", "v", "grad_o")):
        m[k] = far[:, 16 * i:16 * i + 16].view(T, 1, 1, 16)
        m[k].copy_(d[k])
    m.update(g=d["g"].to(gpu_device), beta=d["beta"].to(gpu_device))
    announce("delta steps far")
    seen = [m[k] for k in ("q", "k", "v", "g", "beta")]
    o, last, ckpt = dendsn.delta_rule(cfg, *seen)
    got = dict(o=o, s_last=last, **dendsn.delta_rule_backward(cfg, *seen, None, ckpt, m["grad_o"]))
    for k, (value, bound) in block_ref.delta(d, 0.25, "bf16").items():
        seq_ref.assert_within(got[k], value, bound, k)
