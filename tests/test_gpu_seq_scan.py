"""Gated leaky scan on the GPU against the recurrence in float64."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


def make(T, b, D, io, gate, seed, ragged=False, carry=False):
    gen = torch.Generator().manual_seed(seed)
    dt = seq_ref.io_dtype(io)
    n = lambda *s: torch.randn(s, generator=gen)
    x, g, gh = n(T, b, D).to(dt), 2.0 + 1.5 * n(T, b, D), n(T, b, D).to(dt)
    g = (torch.sigmoid(g) if gate == "decay" else g).to(dt)
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (b,), generator=gen, dtype=torch.int32)
        lengths[0] = 0
        lengths[-1] = T + 7   # clamped
    return dict(x=x, g=g, h0=n(b, D) if carry else None, lengths=lengths, grad_h=gh, grad_last=n(b, D) if carry else None)


def run(cfg, d, dev):
    m = {k: None if v is None else v.to(dev) for k, v in d.items()}
    h, last, ckpt = dendsn.gated_scan(cfg, m["x"], m["g"], m["h0"], m["lengths"])
    out = dict(h=h, h_last=last)
    out.update(dendsn.gated_scan_backward(cfg, m["x"], m["g"], m["lengths"], ckpt, m["grad_h"], m["grad_last"]))
    return out


def check(cfg, d, dev):
    got = run(cfg, d, dev)
    ref = seq_ref.scan(d["x"], d["g"], cfg.gate, cfg.leaky, cfg.io, d["h0"], d["lengths"], d["grad_h"], d["grad_last"])
    for k, (value, bound) in ref.items():
        seq_ref.assert_within(got[k], value, bound, k)
    again = run(cfg, d, dev)
    for k in got:
        assert torch.equal(got[k].contiguous().view(torch.uint8), again[k].contiguous().view(torch.uint8)), k
    return got


# steps around a wave's eight, a tile's 64 and the split of long sequences; channels around a
# wave of one or two a lane
SHAPES = [(1, 1, 1), (1, 3, 64), (2, 1, 65), (7, 2, 130), (8, 1, 2), (9, 3, 63), (63, 1, 128), (64, 2, 66), (65, 1, 127),
          (129, 3, 10), (200, 1, 256), (255, 2, 5), (257, 1, 64), (640, 1, 34), (1000, 2, 7), (2500, 1, 130)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,b,D", SHAPES)
def test_against_recurrence(gpu_device, T, b, D, io):
    for gate, leaky, ragged, carry in (("sigmoid", True, False, False), ("sigmoid", False, True, True),
                                       ("decay", True, True, False), ("decay", False, False, True)):
        cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io, gate=gate, leaky=leaky)
        announce(f"scan {cfg} ragged {ragged} carry {carry}")
        check(cfg, make(T, b, D, io, gate, T + D, ragged, carry), gpu_device)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3, 8, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("b,D", [(3, 1000), (2, 1), (1, 515)])
def test_one_tile(gpu_device, T, b, D, io):
    """Steps around the eight of one, two, four and eight waves, where a block's other waves have
    other channels; rows end inside a block's share."""
    for gate, leaky, ragged, carry in (("sigmoid", True, True, True), ("decay", False, False, False)):
        cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io, gate=gate, leaky=leaky)
        announce(f"scan {cfg} ragged {ragged} carry {carry}")
        check(cfg, make(T, b, D, io, gate, T + D, ragged, carry), gpu_device)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_layouts(gpu_device, io):
    """Batch-major, side by side in one projection, odd strides and broadcast inputs give
    the contiguous call's bits."""
    T, b, D = 150, 3, 24
    cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io)
    d = make(T, b, D, io, "sigmoid", 5, ragged=True, carry=True)
    want = run(cfg, d, gpu_device)

    def same(x, g, gh, what):
        announce(f"scan layout {what} {io}")
        got = run(cfg, dict(d, x=x, g=g, grad_h=gh), gpu_device)
        for k in want:
            # lanes of one or of two channels: the same operations either way
            assert torch.equal(got[k], want[k]), (what, k)

    x, g, gh = (d[k].to(gpu_device) for k in ("x", "g", "grad_h"))
    turn = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    same(turn(x), turn(g), turn(gh), "batch outermost")
    both = torch.cat([x, g], dim=-1)
    same(both[..., :D], both[..., D:], gh, "side by side")
    for pad, at in ((3, 1), (2, 2)):
        wide = torch.full((3, T, b, D + pad), float("nan"), dtype=x.dtype, device=gpu_device)
        for i, t in enumerate((x, g, gh)):
            wide[i, :, :, at:at + D] = t
        same(*(wide[i, :, :, at:at + D] for i in range(3)), f"pad {pad} at {at}")
    one = dict(d, x=d["x"][:1].expand(T, b, D), g=d["g"][:, :1].expand(T, b, D))
    dense = {k: v if v is None else v.contiguous() for k, v in one.items()}
    got, want = run(cfg, one, gpu_device), run(cfg, dense, gpu_device)
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_outputs_with_strides(gpu_device):
    """The entry points with the C names write h, grad_x and grad_g into slices."""
    T, b, D = 70, 2, 10
    cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D)
    d = make(T, b, D, "f32", "sigmoid", 8)
    want = run(cfg, d, gpu_device)
    x, g, gh = (d[k].to(gpu_device) for k in ("x", "g", "grad_h"))
    wide = torch.full((T, b, 3 * D + 1), 7.0, device=gpu_device)
    h, gx, gg = (wide[..., i * D + (i > 1):(i + 1) * D + (i > 1)] for i in range(3))
    ck = torch.empty(dendsn.dendsn_scan_ckpt_bytes(cfg) // 4, device=gpu_device)
    ws = torch.empty(max(16, dendsn.dendsn_scan_workspace_bytes(cfg, True)), dtype=torch.uint8, device=gpu_device)
    announce(f"scan strided outputs {cfg}")
    dendsn.dendsn_scan_forward(cfg, x, g, None, None, h, None, ck, ws)
    dendsn.dendsn_scan_backward(cfg, x, g, None, ck, gh, None, gx, gg, None, ws)
    assert torch.equal(h, want["h"]) and torch.equal(gx, want["grad_x"]) and torch.equal(gg, want["grad_g"])
    assert bool((wide[..., 2 * D] == 7.0).all())


def test_past_the_end_nothing_counts(gpu_device):
    """NaN and infinities at and past a sequence's end change no bit; outputs are +0 there."""
    T, b, D = 300, 4, 12
    for io in ("f32", "bf16"):
        cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io)
        d = make(T, b, D, io, "sigmoid", 9, ragged=True, carry=True)
        d["lengths"] = torch.tensor([0, 1, 129, -3], dtype=torch.int32)
        announce(f"scan padding {cfg}")
        want = run(cfg, d, gpu_device)
        past = torch.arange(T)[:, None, None] >= d["lengths"].clamp(min=0)[None, :, None]
        for bad in (float("nan"), float("inf"), -float("inf")):
            got = run(cfg, dict(d, **{k: torch.where(past, torch.tensor(bad, dtype=d[k].dtype), d[k])
                                      for k in ("x", "g", "grad_h")}), gpu_device)
            for k in want:
                assert torch.equal(got[k].view(torch.uint8), want[k].view(torch.uint8)), (k, bad)
        for k in ("h", "grad_x", "grad_g"):
            assert not want[k].cpu()[past.expand(T, b, D)].view(torch.uint8).any(), k
        assert torch.equal(want["h_last"].cpu()[0], d["h0"][0]) and torch.equal(want["grad_h0"].cpu()[0], d["grad_last"][0])


def test_extreme_gates(gpu_device):
    """Gates of the type's extremes, decays of exactly 0 and 1, and a NaN that only its own
    channel's later steps see."""
    T, b, D = 140, 1, 8
    g = torch.zeros((T, b, D))
    big = torch.finfo(torch.float32).max
    for i, v in enumerate((float("inf"), -float("inf"), big, -big, 88.0, -88.0, 30.0, -30.0)):
        g[:, :, i] = v
    for leaky in (True, False):
        cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, leaky=leaky)
        d = make(T, b, D, "f32", "sigmoid", 2, carry=True)
        announce(f"scan extreme gates {cfg}")
        check(cfg, dict(d, g=g), gpu_device)
    cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, gate="decay")
    d = make(T, b, D, "f32", "decay", 3, carry=True)
    d["g"][:, :, 0], d["g"][:, :, 1], d["g"][::7, :, 2] = 0.0, 1.0, 0.0
    check(cfg, d, gpu_device)
    nan = make(T, b, D, "f32", "decay", 4)
    nan["x"][70, 0, 3] = float("nan")
    check(cfg, nan, gpu_device)


@pytest.mark.parametrize("gate,leaky", [("sigmoid", True), ("sigmoid", False), ("decay", True), ("decay", False)])
def test_gradient_against_differences(gpu_device, gate, leaky):
    """Directional derivatives: central differences of the float64 loss in random directions,
    step 1e-4 (the cubic remainder is below 1e-7 of the derivative's scale), against the
    kernel's gradient, whose own error is within 1e-5 of the summed sizes."""
    T, b, D = 150, 2, 5
    cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, gate=gate, leaky=leaky)
    d = make(T, b, D, "f32", gate, 31, ragged=True, carry=True)
    d["lengths"] = torch.tensor([T, 77], dtype=torch.int32)
    announce(f"scan differences {cfg}")
    got = run(cfg, d, gpu_device)
    f = {k: v.double() for k, v in d.items() if k != "lengths"}
    gen = torch.Generator().manual_seed(1)
    for name, grad in (("x", "grad_x"), ("g", "grad_g"), ("h0", "grad_h0")):
        for _ in range(3):
            v = torch.randn(f[name].shape, generator=gen, dtype=torch.float64)
            at = lambda s: seq_ref.scan_loss(*(f[k] + s * v if k == name else f[k] for k in ("x", "g")), gate, leaky,
                                             f["h0"] + s * v if name == "h0" else f["h0"], d["lengths"], f["grad_h"],
                                             f["grad_last"])
            step = 1e-4
            diff = (at(step) - at(-step)) / (2 * step)
            terms = got[grad].double().cpu() * v
            assert abs(float(terms.sum()) - diff) <= 1e-5 * float(terms.abs().sum()), name


def test_offsets_past_32_bits(gpu_device):
    """Steps that lie 2^27 elements apart."""
    T, b, D = 40, 1, 64
    store = torch.empty(((T - 1) << 27) + D, dtype=torch.bfloat16, device=gpu_device)
    far = store.as_strided((T, b, D), (1 << 27, D, 1))
    cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io="bf16")
    d = make(T, b, D, "bf16", "sigmoid", 6)
    far.copy_(d["x"])
    announce(f"scan far steps {cfg}")
    want, got = run(cfg, d, gpu_device), run(cfg, dict(d, x=far), gpu_device)
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_nothing(gpu_device):
    announce("scan T = 0")
    for h0 in (None, torch.randn(2, 3, device=gpu_device)):
        cfg = dendsn.GatedScanConfig(T=0, batch=2, D=3)
        x = torch.zeros((0, 2, 3), device=gpu_device)
        h, last, ckpt = dendsn.gated_scan(cfg, x, x, h0)
        assert h.shape == (0, 2, 3) and torch.equal(last, torch.zeros_like(last) if h0 is None else h0)
        got = dendsn.gated_scan_backward(cfg, x, x, None, ckpt, x, h0)
        assert torch.equal(got["grad_h0"], last)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("b,D", [(1, 1), (3, 64), (5, 129), (64, 1000), (2, 514)])
def test_step(gpu_device, b, D, io):
    """A token at a time equals the scan; idle requests and held sequences stay as they are."""
    for gate, leaky in (("sigmoid", True), ("decay", False)):
        T, held = 5, b + 3
        cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io, gate=gate, leaky=leaky)
        d = make(T, b, D, io, gate, b + D, carry=True)
        announce(f"scan step {cfg}")
        gen = torch.Generator().manual_seed(2)
        state = torch.randn((held, D), generator=gen)
        slots = torch.randperm(held, generator=gen)[:b].to(torch.int32)
        state[slots.long()] = d["h0"]
        idle = torch.zeros(b, dtype=torch.bool)
        if b > 2:
            idle[1], idle[2] = True, True
            state[slots[1].long()], state[slots[2].long()] = 5.0, 6.0
        on_dev, was = state.to(gpu_device), state.clone()
        given = slots.clone()
        given[idle] = torch.tensor([-1, held], dtype=torch.int32)[:int(idle.sum())]
        ref = seq_ref.scan(d["x"], d["g"], gate, leaky, io, d["h0"])
        one = cfg.with_(T=1)
        x, g = d["x"].to(gpu_device), d["g"].to(gpu_device)
        for t in range(T):
            h = dendsn.gated_scan_step(one, x[t], g[t], on_dev, given.to(gpu_device)).cpu()
            seq_ref.assert_within(h[~idle], ref["h"][0][t][~idle], ref["h"][1][t][~idle], f"h[{t}]")
            assert not h[idle].any()
        now = on_dev.cpu()
        live = slots[~idle].long()
        seq_ref.assert_within(now[live], ref["h_last"][0][~idle], ref["h_last"][1][~idle], "state")
        rest = torch.ones(held, dtype=torch.bool)
        rest[live] = False
        assert torch.equal(now[rest], was[rest])
        # without slots: row b for request b; rows side by side in a projection
        plain = d["h0"].to(gpu_device)
        both = torch.cat([x[0], g[0]], dim=-1)
        h = dendsn.gated_scan_step(one, both[:, :D], both[:, D:], plain)
        seq_ref.assert_within(h, ref["h"][0][0], ref["h"][1][0], "h without slots")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T", [8, 30, 64, 150, 2500])
def test_decays_beyond_one(gpu_device, T, io):
    """Given decays of any size: the product of many is no fp32 number, their states are.  States of
    0 stay 0 until something comes in; a state of 2^-100 is brought up and down again; a decay of 0
    forgets."""
    b, D = 2, 10
    for leaky in (False, True):
        cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io, gate="decay", leaky=leaky)
        d = make(T, b, D, io, "decay", T, carry=True)
        x, g, gh, h0, last = d["x"], d["g"], d["grad_h"], d["h0"], d["grad_last"]
        t = torch.arange(T)
        late = t >= T - T // 4
        # growth while the state is 0: inputs come at the end, gradients at the first step
        for i, a in enumerate((1.25, 2.0 ** 40, -1.5, 2.0 ** 120)):
            g[:, :, i] = torch.where(late, 0.75, a)[:, None]
            x[~late, :, i] = 0.0
            h0[:, i] = 0.0
            last[:, i] = 0.0
            gh[1:, :, i] = 0.0
        # up and down by 2^66 twice
        for i, order in ((4, (66, 66, -66, -66)), (5, (-66, -66, 66, 66))):
            g[:, :, i] = torch.tensor([2.0 ** order[k % 4] for k in range(T)])[:, None]
            x[:, :, i], gh[:, :, i] = 0.0, 0.0
            h0[:, i] = 2.0 ** (-100 if order[0] > 0 else 100)
            # (in range on the way back, and so is its product with the state)
            last[:, i] = 2.0 ** (-100 if order[(T - 1) % 4] > 0 else 100 if T % 4 == 0 else 30)
        # large decays, of which one is 0
        g[:, :, 6] = torch.where(t == T // 2, 0.0, torch.where(t < T // 2, 2.0 ** 30, 0.5))[:, None]
        x[t < T // 2, :, 6], h0[:, 6], gh[:, :, 6], last[:, 6] = 0.0, 0.0, 0.0, 1.0
        # decays far below one, whose product is none either
        g[:, :, 7] = 2.0 ** -100
        announce(f"scan decays beyond one {cfg}")
        check(cfg, d, gpu_device)


@pytest.mark.parametrize("T,b,D,io,gate,leaky,ragged", [
    (700, 16, 2048, "bf16", "sigmoid", True, False), (700, 16, 2048, "f32", "decay", False, True),
    (650, 129, 255, "bf16", "decay", True, True), (650, 129, 255, "f32", "sigmoid", False, False),
    (16400, 1, 2000, "bf16", "sigmoid", True, False), (9000, 2, 1001, "f32", "decay", False, True)])
def test_many_tiles_a_block(gpu_device, T, b, D, io, gate, leaky, ragged):
    """Blocks that walk ten tiles of whole sequences (256 blocks and more: no split), and splits of
    nine tiles a block: every channel is its own recurrence, and some of them are compared."""
    cfg = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io, gate=gate, leaky=leaky)
    d = make(T, b, D, io, gate, T + D, ragged, carry=True)
    announce(f"scan {cfg} ragged {ragged}")
    got, again = run(cfg, d, gpu_device), run(cfg, d, gpu_device)
    some = torch.tensor(sorted({0, 1, 63, 64, 127, 128, 129, D // 2, D - 130, D - 2, D - 1}))
    part = {k: v if v is None or k == "lengths" else v[..., some] for k, v in d.items()}
    ref = seq_ref.scan(part["x"], part["g"], gate, leaky, io, part["h0"], part["lengths"], part["grad_h"],
                       part["grad_last"])
    for k, (value, bound) in ref.items():
        seq_ref.assert_within(got[k].cpu()[..., some], value, bound, k)
    for k in got:
        assert bool(torch.isfinite(got[k]).all()), k
        assert torch.equal(got[k].contiguous().view(torch.uint8), again[k].contiguous().view(torch.uint8)), k
