"""Root-mean-square norm on the GPU against float64."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import block_ref, seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


def rows(n, D, dt, gen, apart=0, std=1.0):
    """[n, D] with ``apart`` values between rows, from an odd place on."""
    flat = (std * torch.randn((n * (D + apart) + 1,), generator=gen)).to(dt)
    return flat[1:].view(n, D + apart)[:, :D] if apart else flat[:n * D].view(n, D)


def make(n, D, io, seed, apart=0):
    gen, dt = torch.Generator().manual_seed(seed), seq_ref.io_dtype(io)
    return dict(x=rows(n, D, dt, gen, apart), residual=rows(n, D, dt, gen, apart, 2.0), weight=(1 + 0.3 * torch.randn((D,), generator=gen)).to(dt),
                grad_y=rows(n, D, dt, gen, apart), grad_sum=rows(n, D, dt, gen, apart))


def on(d, dev):
    out = {}
    for k, v in d.items():  # strides kept
        if v is None or v.dim() == 1:
            out[k] = None if v is None else v.to(dev)
            continue
        ld = v.stride(0) if v.shape[0] > 1 else v.shape[1]
        flat = torch.zeros((v.shape[0] * ld + 1,), dtype=v.dtype, device=dev)
        odd = int(ld != v.shape[1])
        out[k] = flat[odd:odd + v.shape[0] * ld].view(v.shape[0], ld)[:, :v.shape[1]]
        out[k].copy_(v)
    return out


def run(cfg, m, weight, residual):
    w, r = m["weight"] if weight else None, m["residual"] if residual else None
    y, rstd, summed = dendsn.rms_norm(cfg, m["x"], w, r)
    out = dict(y=y, rstd=rstd)
    if residual:
        out["sum"] = summed
    out.update(dendsn.rms_norm_backward(cfg, summed if residual else m["x"], w, rstd, m["grad_y"],
                                        m["grad_sum"] if residual else None))
    return out


# lengths around a pack's 4 and 8, and of 16, 64, 256 and 1024 lanes with four packs each, and past those
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,apart", [(1, 1, 0), (3, 7, 0), (17, 64, 8), (5, 100, 3), (40, 256, 0), (9, 513, 1), (33, 1001, 0),
                                       (70, 2048, 0), (6, 4099, 5), (3, 8192, 0), (2, 16392, 0), (3, 33001, 7)])
def test_against_definition(gpu_device, n, D, apart, io):
    cfg = dendsn.RMSNormConfig(N=n, D=D, io=io, eps=1e-5)
    d = make(n, D, io, n + D, apart)
    m = on(d, gpu_device)
    for weight, residual in ((True, True), (True, False), (False, True), (False, False)):
        announce(f"norm {cfg} weight {weight} residual {residual}")
        got = run(cfg, m, weight, residual)
        ref = block_ref.norm(d["x"], d["weight"] if weight else None, d["residual"] if residual else None, 1e-5, io, d["grad_y"],
                             d["grad_sum"] if residual else None, got["sum"] if residual else None)
        if not weight:
            del ref["grad_weight"]
        assert set(ref) == set(got)
        for k, (value, bound) in ref.items():
            seq_ref.assert_within(got[k], value, bound, k)
        again = run(cfg, m, weight, residual)
        for k in got:
            assert torch.equal(got[k], again[k]), k


def test_many_rows(gpu_device):
    """More rows than the backward's blocks have at once."""
    n, D = 20000, 40
    cfg, d = dendsn.RMSNormConfig(N=n, D=D), make(n, D, "f32", 1)
    announce("norm many rows")
    got = run(cfg, on(d, gpu_device), True, True)
    for k, (value, bound) in block_ref.norm(d["x"], d["weight"], d["residual"], 1e-6, "f32", d["grad_y"], d["grad_sum"], got["sum"]).items():
        seq_ref.assert_within(got[k], value, bound, k)


def test_gradients_against_differences(gpu_device):
    n, D = 6, 50
    cfg, d = dendsn.RMSNormConfig(N=n, D=D), make(n, D, "f32", 2)
    announce("norm differences")
    got = run(cfg, on(d, gpu_device), True, True)
    gen = torch.Generator().manual_seed(3)
    for name, grad in (("x", "grad_x"), ("weight", "grad_weight")):
        way = torch.randn(d[name].shape, generator=gen, dtype=torch.float64)

        def loss(e):
            x = dict(d, **{name: d[name].double() + e * way})
            s = x["x"].double() + x["residual"].double()
            y = s / (s.square().mean(1, keepdim=True) + 1e-6).sqrt() * x["weight"].double()
            return (y * d["grad_y"].double()).sum() + (s * d["grad_sum"].double()).sum()

        slope, mine = (loss(1e-5) - loss(-1e-5)) / 2e-5, (got[grad].double().cpu() * way).sum()
        assert abs(slope - mine) <= 1e-5 * got[grad].double().norm().cpu() * way.norm(), (name, slope, mine)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,apart", [(1, 1, 0), (4, 9, 0), (19, 250, 3), (6, 2048, 0), (3, 5000, 1), (2, 34001, 0)])
def test_e4m3(gpu_device, n, D, apart, io):
    """Rows in 8 bits: the scale is the largest magnitude's 448th part, a value is off by half of e4m3's
    spacing there, and by what y is off by."""
    cfg = dendsn.RMSNormConfig(N=n, D=D, io=io, eps=1e-5)
    d = make(n, D, io, n + D, apart)
    d["x"][n // 2] = 0.0
    d["residual"][n // 2] = 0.0   # a row of zeros
    m = on(d, gpu_device)
    for weight, residual in ((True, True), (False, False)):
        announce(f"norm e4m3 {cfg} {weight}")
        w, r = (m["weight"], m["residual"]) if weight else (None, None)
        y, scale, rstd, summed = dendsn.rms_norm_e4m3(cfg, m["x"], w, r)
        ref = block_ref.norm(d["x"], d["weight"] if weight else None, d["residual"] if residual else None, 1e-5, io)
        seq_ref.assert_within(rstd, *ref["rstd"], "rstd")
        if residual:
            seq_ref.assert_within(summed, *ref["sum"], "sum")
        value = ref["y"][0]
        off = (0.5 * (D + 6) + 10) * seq_ref.U  # of y in fp32
        top = value.abs().amax(1)
        want = torch.where(top > 0, top / 448, 1.0)
        seq_ref.assert_within(scale, want, (off + 2 * seq_ref.U) * want, "scale")
        # (a value at a border may be taken for the other side's: a spacing, not half)
        units = value / want[:, None]
        bound = 0.5 * block_ref.e4m3_spacing(units) + (2 * off + 4 * seq_ref.U) * units.abs() * 2
        seq_ref.assert_within(y.float(), units, bound, "y")


def test_rows_that_are_not_finite(gpu_device):
    """They make no other row so."""
    d = make(5, 300, "f32", 4)
    d["x"][1, 7], d["x"][3, 9] = float("nan"), float("inf")
    m = on(d, gpu_device)
    announce("norm not finite")
    cfg = dendsn.RMSNormConfig(N=5, D=300)
    y, rstd, summed = dendsn.rms_norm(cfg, m["x"], m["weight"], m["residual"])
    assert torch.isfinite(y[[0, 2, 4]]).all() and torch.isnan(y[1]).all() and torch.isnan(y[3, 9])
    y, scale, _, _ = dendsn.rms_norm_e4m3(cfg, m["x"], m["weight"], m["residual"])
    assert torch.isfinite(y[[0, 2, 4]].float()).all() and torch.isnan(y[1, 7].float())


def test_empty(gpu_device):
    cfg = dendsn.RMSNormConfig(N=0, D=10)
    x, w = torch.zeros((0, 10), device=gpu_device), torch.ones((10,), device=gpu_device)
    y, rstd, summed = dendsn.rms_norm(cfg, x, w, x)
    assert y.shape == (0, 10)
    back = dendsn.rms_norm_backward(cfg, x, w, rstd, x)
    assert torch.equal(back["grad_weight"], torch.zeros_like(w))
