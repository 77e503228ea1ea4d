"""The norm's backward from x and the residual, whose sum it forms again in fp32: gradients of the norm of
the sum that the forward had, not of the stored one, which has io's bits."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import block_ref, seq_ref
from tests.parity import announce
from tests.test_gpu_norm import make, on

pytestmark = pytest.mark.gpu


# as the other tests' lengths: every number of lanes and of packs a row, and rows past those kept
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,apart", [(1, 1, 0), (3, 7, 0), (17, 64, 8), (5, 100, 3), (40, 256, 0), (9, 513, 1), (33, 1001, 0),
                                       (70, 2048, 0), (300, 520, 0), (6, 4099, 5), (3, 8192, 0), (2, 16392, 0), (3, 33001, 7)])
def test_against_definition(gpu_device, n, D, apart, io):
    cfg = dendsn.RMSNormConfig(N=n, D=D, io=io, eps=1e-5)
    d = make(n, D, io, n + D, apart)
    m = on(d, gpu_device)
    for weight, grad_sum in ((True, True), (True, False), (False, True)):
        announce(f"norm backward of a residual {cfg} weight {weight} grad_sum {grad_sum}")
        w, gs = m["weight"] if weight else None, m["grad_sum"] if grad_sum else None
        _, rstd, _ = dendsn.rms_norm(cfg, m["x"], w, m["residual"])
        back = lambda: dendsn.rms_norm_backward(cfg, m["x"], w, rstd, m["grad_y"], gs, residual=m["residual"])
        got, again = back(), back()
        ref = block_ref.norm(d["x"], d["weight"] if weight else None, d["residual"], 1e-5, io, d["grad_y"],
                             d["grad_sum"] if grad_sum else None)
        assert set(got) == ({"grad_x", "grad_weight"} if weight else {"grad_x"})
        for k in got:
            seq_ref.assert_within(got[k], *ref[k], k)
            assert torch.equal(got[k], again[k]), k


def test_the_stored_sum_is_off_by_its_rounding(gpu_device):
    """What the sum's rounding to bf16 costs grad_weight, a sum over rows that fall either way: beside the
    result's own rounding (half a step at most, 2^-8 of each value) another of hat's."""
    n, D = 4096, 512
    cfg, d = dendsn.RMSNormConfig(N=n, D=D, io="bf16"), make(n, D, "bf16", 5)
    m = on(d, gpu_device)
    announce("norm backward, both forms")
    _, rstd, summed = dendsn.rms_norm(cfg, m["x"], m["weight"], m["residual"])
    want = block_ref.norm(d["x"], d["weight"], d["residual"], 1e-6, "bf16", d["grad_y"])["grad_weight"][0]
    off = {}
    for name, x, r in (("stored", summed, None), ("formed", m["x"], m["residual"])):
        got = dendsn.rms_norm_backward(cfg, x, m["weight"], rstd, m["grad_y"], residual=r)["grad_weight"].double().cpu()
        off[name] = float((got - want).norm() / want.norm())
    print(off, flush=True)
    rounding = float((want.to(torch.bfloat16).double() - want).norm() / want.norm())
    assert off["formed"] <= 1.01 * rounding < off["stored"]


def test_a_row_for_all_and_empty(gpu_device):
    """A residual that is one row (stride 0); no rows; a residual of another shape is refused."""
    cfg, d = dendsn.RMSNormConfig(N=9, D=40), make(9, 40, "f32", 6)
    m = on(d, gpu_device)
    one = m["residual"][:1].expand(9, 40)
    announce("norm backward, residual broadcast")
    _, rstd, _ = dendsn.rms_norm(cfg, m["x"], m["weight"], one)
    got = dendsn.rms_norm_backward(cfg, m["x"], m["weight"], rstd, m["grad_y"], residual=one)
    ref = block_ref.norm(d["x"], d["weight"], d["residual"][:1].expand(9, 40), 1e-6, "f32", d["grad_y"])
    for k in got:
        seq_ref.assert_within(got[k], *ref[k], k)
    none = cfg.with_(N=0)
    got = dendsn.rms_norm_backward(none, m["x"][:0], m["weight"], rstd[:0], m["grad_y"][:0], residual=one[:0])
    assert got["grad_x"].shape == (0, 40) and not got["grad_weight"].any()
    with pytest.raises(ValueError):
        dendsn.rms_norm_backward(cfg, m["x"], m["weight"], rstd, m["grad_y"], residual=one[:8])


def test_squares_past_fp32(gpu_device):
    """As documented: a row whose squares' sum passes fp32 has an rstd and a y of 0, the others their own."""
    d = make(4, 96, "f32", 7)
    d["x"][2] = 1e20
    m = on(d, gpu_device)
    announce("norm of squares past fp32")
    cfg = dendsn.RMSNormConfig(N=4, D=96)
    y, rstd, _ = dendsn.rms_norm(cfg, m["x"], m["weight"])
    assert float(rstd[2]) == 0 and not y[2].any()
    ref = block_ref.norm(d["x"], d["weight"], None, 1e-6, "f32")["y"]
    keep = [0, 1, 3]
    seq_ref.assert_within(y[keep], ref[0][keep], ref[1][keep], "y")
