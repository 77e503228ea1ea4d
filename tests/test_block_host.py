"""Host-side checks of include/dendsn_block.h: exports, sizes, and every refusal.

Nothing here touches a GPU: each call queries a size, is of no elements, or fails the
argument checks, which run on the host before any launch.
"""

import ctypes
import os
import re

import pytest
import torch

import paper_2412_06355_amd as dendsn
from paper_2412_06355_amd.block import dendsn_adamw_cfg, dendsn_adamw_tensor, dendsn_delta_cfg, dendsn_norm_cfg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
A = 0x10000          # an aligned address
BIG = 1 << 46


@pytest.fixture(scope="module")
def lib():
    return dendsn.block_lib()


def ref(cfg):
    return ctypes.byref(cfg) if cfg is not None else None


def p(v):
    return None if v is None else ctypes.c_void_p(v)


def test_every_declared_function_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "dendsn_block.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(dendsn_[a-z0-9_]+)\s*\(", text))
    assert declared == set(dendsn.BLOCK_EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


# -- delta rule ----------------------------------------------------------------
def delta_cfg(**kw):
    c = dict(T=10, batch=2, H=4, Hk=2, K=16, V=24, io=0, scale=1.0)
    for n, row in (("q", 32), ("k", 32), ("v", 96), ("g", 4), ("beta", 4), ("o", 96), ("grad_o", 96)):
        c.update({f"{n}_t": 2 * row, f"{n}_b": row, f"{n}_h": row // (2 if n in "qk" else 4)})
    c.update(kw)
    return dendsn_delta_cfg(**c)


def delta_fwd(lib, c, nbytes=1 << 40, **kw):
    a = dict(q=A, k=2 * A, v=3 * A, g=4 * A, beta=5 * A, s0=None, lengths=None, o=6 * A, s_last=None, ckpt=None, ws=7 * A)
    a.update(kw)
    return lib.dendsn_delta_forward(ref(c), *(p(x) for x in a.values()), nbytes, None)


def delta_bwd(lib, c, nbytes=1 << 40, **kw):
    a = dict(q=A, k=2 * A, v=3 * A, g=4 * A, beta=5 * A, lengths=None, ckpt=8 * A, grad_o=6 * A, grad_s_last=None, gq=9 * A,
             gk=10 * A, gv=11 * A, gg=12 * A, gbeta=13 * A, gs0=None, ws=7 * A)
    a.update(kw)
    return lib.dendsn_delta_backward(ref(c), *(p(x) for x in a.values()), nbytes, None)


def delta_step(lib, c, n_slots=8, slots=8 * A, state=7 * A, **kw):
    a = dict(q=A, k=2 * A, v=3 * A, g=4 * A, beta=5 * A)
    o = kw.pop("o", 6 * A)
    a.update(kw)
    return lib.dendsn_delta_step(ref(c), *(p(x) for x in a.values()), n_slots, p(slots), p(state), p(o), None)


@pytest.mark.parametrize("kw", [
    dict(T=-1), dict(T=(1 << 24) + 1), dict(batch=-1), dict(batch=65536), dict(H=-1), dict(H=65536), dict(Hk=0), dict(Hk=3),
    dict(Hk=-2), dict(K=0), dict(V=0), dict(V=65537), dict(io=2), dict(io=-1), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(q_t=-1), dict(k_b=BIG + 1), dict(v_h=-4), dict(g_t=1 << 45), dict(beta_h=-1),
    dict(o_t=-1), dict(grad_o_b=-1), dict(T=1 << 24, batch=65535, H=65532, V=65536)])
def test_delta_bad_cfg(lib, kw):
    c, out = delta_cfg(**kw), ctypes.c_size_t(77)
    assert lib.dendsn_delta_ckpt_bytes(ref(c), ctypes.byref(out)) == INVALID and out.value == 77
    assert lib.dendsn_delta_workspace_bytes(ref(c), 1, ctypes.byref(out)) == INVALID and out.value == 77
    assert delta_fwd(lib, c) == INVALID and delta_bwd(lib, c) == INVALID and delta_step(lib, c) == INVALID
    assert dendsn.dendsn_seq_last_error() != ""


def test_delta_unsupported(lib):
    c = delta_cfg(K=129)
    assert delta_fwd(lib, c) == UNSUPPORTED and delta_bwd(lib, c) == UNSUPPORTED
    assert delta_step(lib, delta_cfg(K=129, T=1)) == UNSUPPORTED
    # steps that lie too far apart, more blocks than a launch has (a step has its own)
    assert delta_step(lib, delta_cfg(batch=65535, H=256, Hk=2, K=1, V=1, T=1), slots=None) == INVALID
    for kw in (dict(k_t=1 << 24), dict(io=1, grad_o_t=1 << 25), dict(batch=65535, H=64, Hk=2, V=128, T=2),
               dict(batch=65535, H=256, Hk=2, K=1, V=1, T=1)):
        assert delta_fwd(lib, delta_cfg(**kw)) == UNSUPPORTED, kw


def test_delta_arguments(lib):
    c = delta_cfg()
    assert delta_fwd(lib, None) == INVALID and delta_bwd(lib, None) == INVALID and delta_step(lib, None) == INVALID
    assert lib.dendsn_delta_ckpt_bytes(ref(c), None) == INVALID
    for k in ("q", "k", "v", "g", "beta", "o"):
        assert delta_fwd(lib, c, **{k: None}) == INVALID
        assert delta_fwd(lib, c, **{k: A + 2}) == INVALID
    for k in ("s0", "lengths", "s_last"):
        assert delta_fwd(lib, c, **{k: A + 2}) == INVALID
    assert delta_fwd(lib, c, ckpt=A + 8) == INVALID
    for k in ("q", "k", "v", "g", "beta", "grad_o", "ckpt", "gq", "gk", "gv", "gg", "gbeta"):
        assert delta_bwd(lib, c, **{k: None}) == INVALID
        assert delta_bwd(lib, c, **{k: A + 2}) == INVALID
    for k in ("grad_s_last", "lengths", "gs0"):
        assert delta_bwd(lib, c, **{k: A + 2}) == INVALID
    need = ctypes.c_size_t(0)
    for back, call in ((0, delta_fwd), (1, delta_bwd)):
        assert lib.dendsn_delta_workspace_bytes(ref(c), back, ctypes.byref(need)) == OK and need.value > 0
        assert call(lib, c, nbytes=need.value - 1) == WORKSPACE
        assert call(lib, c, ws=None) == WORKSPACE and call(lib, c, ws=A + 8) == WORKSPACE
    # rows of o that overlap, whichever dimension steps over too little
    for kw in (dict(o_h=23), dict(o_b=95), dict(o_t=191), dict(o_t=0), dict(o_b=0)):
        assert delta_fwd(lib, delta_cfg(**kw)) == INVALID, kw


def test_delta_step_arguments(lib):
    c = delta_cfg(T=1)
    assert delta_step(lib, delta_cfg(T=2)) == INVALID
    for k in ("q", "k", "v", "g", "beta", "o"):
        assert delta_step(lib, c, **{k: None}) == INVALID
        assert delta_step(lib, c, **{k: A + 1}) == INVALID
    assert delta_step(lib, c, state=None) == INVALID and delta_step(lib, c, state=A + 2) == INVALID
    assert delta_step(lib, c, slots=A + 2) == INVALID and delta_step(lib, c, n_slots=-1) == INVALID
    assert delta_step(lib, c, n_slots=1, slots=None) == INVALID
    assert delta_step(lib, delta_cfg(T=1, batch=0)) == OK
    assert delta_step(lib, delta_cfg(T=1, o_h=20)) == INVALID


def test_delta_empty_needs_nothing(lib):
    for kw in (dict(T=0), dict(batch=0), dict(H=0)):
        c, out = delta_cfg(**kw), ctypes.c_size_t(77)
        assert lib.dendsn_delta_ckpt_bytes(ref(c), ctypes.byref(out)) == OK and out.value == 0
        none = {k: None for k in ("q", "k", "v", "g", "beta")}
        assert delta_fwd(lib, c, nbytes=0, ws=None, o=None, **none) == OK
        assert delta_fwd(lib, delta_cfg(H=0, Hk=0), nbytes=0, ws=None, o=None, **none) == OK
        assert delta_bwd(lib, c, nbytes=0, ws=None, ckpt=None, grad_o=None, gq=None, gk=None, gv=None, gg=None, gbeta=None, **none) == OK


# -- norm ------------------------------------------------------------------------
def norm_cfg(**kw):
    c = dict(N=10, D=64, ld_x=64, ld_residual=64, ld_y=64, ld_sum=64, ld_grad_y=64, ld_grad_sum=64, ld_grad_x=64, io=0, eps=1e-6)
    c.update(kw)
    return dendsn_norm_cfg(**c)


def norm_fwd(lib, c, x=A, residual=2 * A, weight=3 * A, y=4 * A, s=5 * A, rstd=6 * A):
    return lib.dendsn_norm_forward(ref(c), p(x), p(residual), p(weight), p(y), p(s), p(rstd), None)


def norm_e4m3(lib, c, x=A, residual=2 * A, weight=3 * A, y=4 * A, scale=7 * A, s=5 * A, rstd=6 * A):
    return lib.dendsn_norm_forward_e4m3(ref(c), p(x), p(residual), p(weight), p(y), p(scale), p(s), p(rstd), None)


def norm_bwd(lib, c, x=A, weight=2 * A, rstd=3 * A, gy=4 * A, gs=5 * A, gx=6 * A, gw=7 * A, ws=8 * A, nbytes=1 << 40):
    return lib.dendsn_norm_backward(ref(c), p(x), p(weight), p(rstd), p(gy), p(gs), p(gx), p(gw), p(ws), nbytes, None)


@pytest.mark.parametrize("kw", [
    dict(N=-1), dict(N=1 << 31), dict(D=0), dict(D=(1 << 22) + 1), dict(io=2), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(ld_x=-1), dict(ld_residual=BIG), dict(ld_y=63), dict(ld_sum=0), dict(ld_grad_y=-1),
    dict(ld_grad_sum=-1), dict(ld_grad_x=63)])
def test_norm_bad_cfg(lib, kw):
    c, out = norm_cfg(**kw), ctypes.c_size_t(77)
    assert lib.dendsn_norm_workspace_bytes(ref(c), ctypes.byref(out)) == INVALID and out.value == 77
    assert norm_fwd(lib, c) == INVALID and norm_e4m3(lib, c) == INVALID and norm_bwd(lib, c) == INVALID


def test_norm_arguments(lib):
    c = norm_cfg()
    for f in (norm_fwd, norm_e4m3, norm_bwd):
        assert f(lib, None) == INVALID
    for k in ("x", "y"):
        assert norm_fwd(lib, c, **{k: None}) == INVALID and norm_e4m3(lib, c, **{k: None}) == INVALID
    assert norm_e4m3(lib, c, scale=None) == INVALID and norm_e4m3(lib, c, scale=A + 2) == INVALID
    for k in ("x", "residual", "weight", "y", "s", "rstd"):
        assert norm_fwd(lib, c, **{k: A + 2}) == INVALID
    for k in ("x", "rstd", "gy", "gx", "gw"):
        assert norm_bwd(lib, c, **{k: None}) == INVALID
    for k in ("x", "weight", "rstd", "gy", "gs", "gx", "gw"):
        assert norm_bwd(lib, c, **{k: A + 2}) == INVALID
    need = ctypes.c_size_t(0)
    assert lib.dendsn_norm_workspace_bytes(ref(c), ctypes.byref(need)) == OK and need.value > 0
    assert norm_bwd(lib, c, nbytes=need.value - 1) == WORKSPACE and norm_bwd(lib, c, ws=None) == WORKSPACE
    assert norm_fwd(lib, norm_cfg(N=0), x=None, y=None) == OK
    assert norm_bwd(lib, norm_cfg(N=0), x=None, rstd=None, gy=None, gx=None, weight=None, gw=None) == OK
    long = norm_cfg(N=(1 << 23) + 1, D=8192, **{k: 8192 for k in ("ld_x", "ld_residual", "ld_y", "ld_sum", "ld_grad_y",
                                                                  "ld_grad_sum", "ld_grad_x")})
    assert norm_fwd(lib, long) == UNSUPPORTED


# -- AdamW -----------------------------------------------------------------------
def adamw_cfg(**kw):
    c = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, state=0)
    c.update(kw)
    return dendsn_adamw_cfg(**c)


def tensor(**kw):
    t = dict(n=100, param=A, grad=2 * A, m=3 * A, v=4 * A, m_scale=5 * A, v_scale=6 * A, copy=7 * A, grad_io=0)
    t.update(kw)
    return dendsn_adamw_tensor(**t)


def adamw(lib, c, tensors=(), count=None, step=1, step_dev=None, scale=None):
    array = (dendsn_adamw_tensor * max(1, len(tensors)))(*tensors)
    return lib.dendsn_adamw_step(ref(c), ctypes.cast(array, ctypes.c_void_p), len(tensors) if count is None else count,
                                 step, p(step_dev), p(scale), 0, None)


@pytest.mark.parametrize("kw", [
    dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")),
    dict(eps=-1e-8), dict(eps=float("inf")), dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(state=2), dict(state=-1)])
def test_adamw_bad_cfg(lib, kw):
    assert adamw(lib, adamw_cfg(**kw)) == INVALID


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(n=(1 << 34) + 1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=A + 2),
    dict(grad=A + 2), dict(grad=A + 1, grad_io=1), dict(m=A + 2), dict(v=A + 1), dict(copy=A + 1), dict(m_scale=A + 2),
    dict(grad_io=2)])
def test_adamw_bad_tensor(lib, kw):
    """Anywhere in the list, and before any launch."""
    assert adamw(lib, adamw_cfg(), [tensor(n=0), tensor(**kw)]) == INVALID
    assert "tensor 1" in dendsn.dendsn_seq_last_error()


def test_adamw_arguments(lib):
    c = adamw_cfg()
    assert adamw(lib, None) == INVALID
    assert adamw(lib, c, count=-1) == INVALID and adamw(lib, c, count=(1 << 20) + 1) == INVALID
    assert lib.dendsn_adamw_step(ref(c), None, 1, 1, None, None, 0, None) == INVALID
    for step in (0, -1, 1 << 31):
        assert adamw(lib, c, step=step) == INVALID
    assert adamw(lib, c, step_dev=A + 2) == INVALID and adamw(lib, c, scale=A + 1) == INVALID
    for k in ("m_scale", "v_scale"):
        assert adamw(lib, adamw_cfg(state=1), [tensor(**{k: None})]) == INVALID
    assert adamw(lib, c) == OK and adamw(lib, c, [tensor(n=0, param=None, grad=None, m=None, v=None)] * 50) == OK


# -- the binding -------------------------------------------------------------------
def test_binding_refuses():
    """Shapes, types, layouts and tensors of the CPU."""
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)
    cfg = dendsn.DeltaRuleConfig(T=4, batch=2, H=2, K=8, V=6)
    good = dict(q=z(4, 2, 2, 8), k=z(4, 2, 2, 8), v=z(4, 2, 2, 6), g=z(4, 2, 2), beta=z(4, 2, 2))
    for name, bad in (("q", z(4, 2, 2, 7)), ("k", z(4, 2, 1, 8)), ("v", z(4, 2, 2, 6, dt=torch.bfloat16)), ("g", z(4, 2)),
                      ("beta", z(4, 2, 2, dt=torch.bfloat16)), ("q", z(4, 2, 8, 2).transpose(2, 3)), ("k", None), ("g", None)):
        with pytest.raises((ValueError, AttributeError)):
            dendsn.delta_rule(cfg, **dict(good, **{name: bad}))
    with pytest.raises(ValueError):
        dendsn.delta_rule(cfg, **good)  # of the CPU
    n = dendsn.RMSNormConfig(N=3, D=4)
    for kw in (dict(x=z(3, 5)), dict(x=z(3, 4), weight=z(5)), dict(x=z(3, 4), residual=z(2, 4)), dict(x=z(3, 4))):
        with pytest.raises(ValueError):
            dendsn.rms_norm(n, **kw)
    a, one = dendsn.AdamWConfig(), [z(4)]
    state = [(z(4), z(4))]
    for args in ((one, [], state), (one, [z(5)], state), (one, one, [(z(4),)]), ([z(4, dt=torch.bfloat16)], one, state),
                 (one, [z(4, dt=torch.float16)], state), (one, [z(8)[::2]], state), (one, one, state)):
        with pytest.raises(ValueError):
            dendsn.adamw(a, *args, 1)
    with pytest.raises(ValueError, match="twice"):
        dendsn.adamw(a, one * 2, [z(4), z(4)], state * 2, 1)
    dendsn.adamw(a, [], [], [], 1)
