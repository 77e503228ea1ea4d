"""The AdamW step on the GPU against float64, and its 8-bit states."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import block_ref, seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu

# sizes around a lane's 4, a wave's (and a scale's) 256 and a block's 8192
SIZES = [1, 3, 4, 5, 0, 255, 256, 257, 1021, 8191, 8192, 8195, 20000]


def make(sizes, seed, dev, grads=torch.float32, packed=True):
    """Tensors packed one after another (so that most start at no multiple of 16 bytes)."""
    gen = torch.Generator().manual_seed(seed)
    total = sum(sizes)
    cut = lambda flat: [t.to(dev) for t in flat.split(sizes)] if not packed else list(flat.to(dev).split(sizes))
    n = lambda std: std * torch.randn((total,), generator=gen)
    return cut(n(0.05)), cut(n(1e-2).to(grads)), cut(n(3e-3)), cut(n(1e-2).square())


@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16])
def test_against_formula(gpu_device, grads):
    p, g, m, v = make(SIZES, 1, gpu_device, grads)
    copies = [torch.zeros(x.shape, dtype=torch.bfloat16, device=gpu_device) if i % 3 else None for i, x in enumerate(p)]
    cfg = dendsn.AdamWConfig(lr=2e-3, beta1=0.85, beta2=0.99, eps=1e-6, weight_decay=0.1)
    scale = torch.tensor([0.5], device=gpu_device)
    want = [block_ref.adamw(*x, 7, 2e-3, 0.85, 0.99, 1e-6, 0.1, 0.5) for x in zip(p, g, m, v)]
    announce(f"adamw {grads}")
    dendsn.adamw(cfg, p, g, list(zip(m, v)), 7, copies=copies, grad_scale=scale)
    for i, ref in enumerate(want):
        for name, got in (("p", p[i]), ("m", m[i]), ("v", v[i])):
            seq_ref.assert_within(got, *ref[name], f"{name} of {SIZES[i]}")
        if copies[i] is not None:
            assert torch.equal(copies[i], p[i].to(torch.bfloat16))


def test_many_tensors(gpu_device):
    """More tensors than a launch takes, empty ones among them."""
    sizes = [(37 * i) % 700 if i % 5 else 0 for i in range(211)]
    p, g, m, v = make(sizes, 2, gpu_device)
    want = [block_ref.adamw(*x, 1) for x in zip(p, g, m, v)]
    announce("adamw many")
    dendsn.adamw(dendsn.AdamWConfig(), p, g, list(zip(m, v)), 1)
    for i, ref in enumerate(want):
        for name, got in (("p", p[i]), ("m", m[i]), ("v", v[i])):
            seq_ref.assert_within(got, *ref[name], f"{name} of tensor {i}")


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_step_on_the_device(gpu_device, state):
    """A step's number on the device gives what the same number on the host does, to the rounding of
    the corrections; the random bits are the same."""
    cfg = dendsn.AdamWConfig(state=state)
    announce(f"adamw device step {state}")
    out = []
    for step in (12, torch.tensor([12], dtype=torch.int32, device=gpu_device)):
        p, g, _, _ = make([1000, 37], 3, gpu_device)
        states = dendsn.adamw_states(cfg, p)
        for _ in range(2):
            dendsn.adamw(cfg, p, g, states, step, seed=5)
        out.append((p, states))
    for a, b in zip(*[x[0] for x in out]):
        assert float((a - b).abs().max()) <= 1e-6 * float(a.abs().max())
    if state == "e4m3":
        for a, b in zip(*[x[1] for x in out]):
            assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8))


def decoded(codes, scales):
    n = codes.numel()
    return codes.float() * scales.repeat_interleave(256)[:n]


def test_8bit_states(gpu_device):
    """One step from 8-bit states: the parameters follow from the values held; new states lie at one of
    the two neighbours of the exact ones, in units of the block's largest."""
    cfg = dendsn.AdamWConfig(state="e4m3", weight_decay=0.1)
    p, g, _, _ = make(SIZES, 4, gpu_device)
    states = dendsn.adamw_states(cfg, p)
    announce("adamw 8 bits")
    for step in (1, 2, 3):
        held = [(decoded(s[0], s[1]), decoded(s[2], s[3]).double().square()) for s in states]
        want = [block_ref.adamw(a, b, m, v, step, wd=0.1) for a, b, (m, v) in zip(p, g, held)]
        dendsn.adamw(cfg, p, g, states, step, seed=9)
        for i, ref in enumerate(want):
            if SIZES[i] == 0:
                continue
            seq_ref.assert_within(p[i], *ref["p"], f"p of {SIZES[i]}")
            for (codes, scales), x in ((states[i][:2], ref["m"][0]), (states[i][2:], ref["v"][0].sqrt())):
                blocks = torch.nn.functional.pad(x.abs(), (0, -x.numel() % 256)).view(-1, 256).amax(1)
                unit = torch.where(blocks > 0, blocks / 448, 1.0)
                seq_ref.assert_within(scales, unit, 20 * seq_ref.U * unit, "scale")
                units = x / unit.repeat_interleave(256)[:x.numel()]
                # at most a spacing away; from 16/16ths of it on where fp32 rounds over a border
                away = (codes.double().cpu() - units).abs()
                assert bool((away <= block_ref.e4m3_spacing(units) * (1 + 2 ** -10)).all()), (SIZES[i], step)
            assert bool((states[i][2].float().cpu()[ref["v"][0] > 0] > 0).all())


def test_rounding_keeps_the_mean(gpu_device):
    """v decays by a thousandth a step with gradients of 0, and in 8 bits its root's mean does too: of n
    values, each off by at most a sixteenth of itself a step at random, the mean over n = 2^18
    is off by at most 6 sqrt(steps / n) / 16."""
    n, steps = 1 << 18, 50
    cfg = dendsn.AdamWConfig(state="e4m3")
    p, g = torch.zeros(n, device=gpu_device), torch.zeros(n, device=gpu_device)
    gen = torch.Generator().manual_seed(6)
    (m, ms, r, rs), = dendsn.adamw_states(cfg, [p])
    r.copy_((100 + 300 * torch.rand((n,), generator=gen)).to(torch.float8_e4m3fn))
    r.view(-1, 256)[:, 0] = 448.0
    first = r.float().mean()
    announce("adamw mean")
    for step in range(1, steps + 1):
        dendsn.adamw(cfg, [p], [g], [(m, ms, r, rs)], step, seed=step)
    held = decoded(r, rs).mean()
    want = first * 0.999 ** (steps / 2)
    assert abs(float(held / want) - 1) <= 6 * (steps / n) ** 0.5 / 16 + 1e-5
    assert float(held) < 0.99 * float(first)


def test_seeds_differ_and_repeat(gpu_device):
    cfg = dendsn.AdamWConfig(state="e4m3")
    announce("adamw seeds")

    def once(seed):
        p, g, _, _ = make([5000, 5000], 7, gpu_device)
        g[1].copy_(g[0])
        states = dendsn.adamw_states(cfg, p)
        dendsn.adamw(cfg, p, g, states, 1, seed=seed)
        return [s[0].view(torch.uint8) for s in states]

    a, b, c = once(1), once(1), once(1 + (1 << 40))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert not torch.equal(a[0], c[0]) and not torch.equal(a[0], a[1])


@pytest.mark.parametrize("eps", [1e-40, 1e-300])
def test_eps_below_the_normal_numbers(gpu_device, eps):
    """Values that have had no gradient stay as they are: 0 / (0 + eps) is 0."""
    p, g, m, v = make([600], 8, gpu_device)
    for t in (g[0], m[0], v[0]):
        t[:300] = 0
    before = p[0].clone()
    cfg = dendsn.AdamWConfig(lr=1e-3, eps=eps, weight_decay=0.0)
    want = block_ref.adamw(before, g[0], m[0], v[0], 3, lr=1e-3, eps=eps, wd=0.0)
    announce(f"adamw eps {eps}")
    dendsn.adamw(cfg, p, g, [(m[0], v[0])], 3)
    assert torch.equal(p[0][:300], before[:300])
    seq_ref.assert_within(p[0][300:], *(x[300:] for x in want["p"]), "p")


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_gradients_that_are_not_finite(gpu_device, state):
    """NaN stays with its value; infinity does too, but for 8-bit states, whose block it takes."""
    cfg = dendsn.AdamWConfig(state=state)

    def once(at):
        p, g, _, _ = make([1100], 9, gpu_device)
        g[0][[300, 600]] = 0.0
        for i, x in at:
            g[0][i] = x
        states = dendsn.adamw_states(cfg, p)
        dendsn.adamw(cfg, p, g, states, 1, seed=5)
        return [p[0]] + [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in states[0]], states[0]

    announce(f"adamw not finite {state}")
    (want, _), (got, held) = once([]), once([(300, float("nan")), (600, float("inf"))])
    place = torch.arange(1100, device=gpu_device)
    own, block = (place == 300) | (place == 600), (place == 300) | (place // 256 == 2)
    assert not got[0][own].isfinite().any() and torch.equal(got[0][~own], want[0][~own])
    codes = (1, 2) if state == "f32" else (1, 3)
    for i in codes:
        spared = ~own if state == "f32" else ~block
        assert torch.equal(got[i][spared], want[i][spared])
        assert not held[i - 1].float()[own].isfinite().any()
    if state == "e4m3":
        for i in (2, 4):
            assert torch.equal(got[i][[0, 1, 3, 4]], want[i][[0, 1, 3, 4]])
