"""What the block operators refuse, and what they do not, without a GPU: the binding's tensors are of the
CPU, so that a call that is not refused for its arguments is refused for where they lie; a C call that
is not refused for its sizes is for an address."""

import ctypes

import pytest
import torch

import paper_2412_06355_amd as dendsn
from paper_2412_06355_amd.block import dendsn_norm_cfg


def adamw_lists(state, copies=True):
    n = (300, 5)
    cfg = dendsn.AdamWConfig(state=state)
    params = [torch.zeros(k) for k in n]
    return cfg, dict(params=params, grads=[torch.zeros(k) for k in n], states=dendsn.adamw_states(cfg, params),
                     copies=[torch.zeros(k, dtype=torch.bfloat16) for k in n] if copies else None)


def refusal(cfg, lists):
    with pytest.raises(ValueError) as e:
        dendsn.adamw(cfg, lists["params"], lists["grads"], lists["states"], 1, copies=lists["copies"])
    return str(e.value)


@pytest.mark.parametrize("state,part", [("f32", 0), ("f32", 1), ("e4m3", 0), ("e4m3", 1), ("e4m3", 2), ("e4m3", 3)])
def test_a_state_that_two_tensors_share(state, part):
    """Each part of a state, of two tensors of one size: two blocks of one launch would write it."""
    cfg, x = adamw_lists(state)
    x.update({k: [v[0], v[0].clone()] if k in ("params", "grads", "copies") else v for k, v in x.items()})
    one = [t.clone() for t in x["states"][0]]
    two = [t.clone() for t in one]
    x["states"] = [one, two]
    assert "twice" not in refusal(cfg, x)
    two[part] = one[part]
    assert "twice" in refusal(cfg, x)


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_arrays_of_one_tensor_that_are_one(state):
    cfg, x = adamw_lists(state)
    assert "twice" not in refusal(cfg, x)
    s = x["states"][0]
    half = len(s) // 2
    x["states"][0] = (*s[:half], *s[:half])  # v is m, and with it its scale
    assert "twice" in refusal(cfg, x)


def test_copies_and_parameters():
    cfg, x = adamw_lists("f32")
    x["params"][1] = torch.zeros(300)
    x["grads"][1] = x["grads"][0]        # read alone: may be shared
    x["states"][1] = tuple(torch.zeros(300) for _ in range(2))
    x["copies"][1] = torch.zeros(300, dtype=torch.bfloat16)
    assert "twice" not in refusal(cfg, x)
    assert "twice" in refusal(cfg, dict(x, copies=[x["copies"][0]] * 2))
    assert "twice" in refusal(cfg, dict(x, copies=[x["params"][0].view(torch.bfloat16)[:300], None]))
    assert "twice" in refusal(cfg, dict(x, states=[(x["params"][1], torch.zeros(300)), x["states"][1]]))
    assert "twice" in refusal(cfg, dict(x, params=[x["params"][0]] * 2))


def test_empty_tensors_are_no_arrays():
    cfg, x = adamw_lists("f32", copies=False)
    for k in ("params", "grads"):
        x[k] += [torch.zeros(0)] * 2
    x["states"] += [(torch.zeros(0), torch.zeros(0))] * 2
    assert "twice" not in refusal(cfg, x)


def norm_call(e4m3=False, x=0x10001, **kw):
    """The status of a norm's forward whose x is misaligned (INVALID), if its size is not refused before."""
    c = dict(N=10, D=64, io=0, eps=1e-6)
    c.update(kw)
    for k in ("ld_x", "ld_residual", "ld_y", "ld_sum", "ld_grad_y", "ld_grad_sum", "ld_grad_x"):
        c.setdefault(k, c["D"])
    call = dendsn.block_lib().dendsn_norm_forward_e4m3 if e4m3 else dendsn.block_lib().dendsn_norm_forward
    at = [ctypes.c_void_p(a) for a in (x, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, 0x70000)[:7 if e4m3 else 6]]
    return call(ctypes.byref(dendsn_norm_cfg(**c)), *at, None)


def test_norm_rows_that_memory_holds_are_not_refused():
    """Many long rows: in 8 bits, or of an x whose rows are one or overlap.  What x and y span together
    is the limit, whatever a row's length."""
    INVALID, UNSUPPORTED, many = 1, 2, (1 << 23) + 1
    assert norm_call(e4m3=True, N=many, D=8200, io=1) == INVALID              # 128 + 64 GiB
    assert norm_call(e4m3=True, N=many, D=16384, io=1, ld_x=0) == INVALID     # 128 GiB of y
    assert norm_call(N=many, D=8200, io=1, ld_x=1) == INVALID
    assert norm_call(N=1 << 24, D=4096) == INVALID                            # 2^39 bytes, all of them
    assert norm_call(N=1 << 23, D=8192) == INVALID
    assert norm_call(N=many, D=8192) == UNSUPPORTED
    assert norm_call(N=(1 << 24) + 1, D=4096) == UNSUPPORTED
    assert norm_call(N=0, D=1 << 22) == INVALID


def test_norm_backward_of_a_residual():
    c = dict(N=10, D=64, io=0, eps=1e-6, **{k: 64 for k in ("ld_x", "ld_residual", "ld_y", "ld_sum", "ld_grad_y", "ld_grad_sum",
                                                            "ld_grad_x")})

    def call(ws=0x90000, nbytes=1 << 40, n=10, **kw):
        at = dict(x=0x10000, residual=0x20000, weight=0x30000, rstd=0x40000, grad_y=0x50000, grad_sum=None, grad_x=0x60000,
                  grad_weight=0x70000)
        at.update(kw)
        return dendsn.block_lib().dendsn_norm_backward_residual(
            ctypes.byref(dendsn_norm_cfg(**dict(c, N=n))), *(ctypes.c_void_p(a) for a in at.values()), ctypes.c_void_p(ws), nbytes, None)

    for k in ("x", "rstd", "grad_y", "grad_x", "grad_weight"):
        assert call(**{k: None}) == 1, k
    for k in ("x", "residual", "weight", "rstd", "grad_y", "grad_sum", "grad_x", "grad_weight"):
        assert call(**{k: 0x10002}) == 1, k
    assert call(ws=None) == 3 and call(nbytes=4) == 3 and call(ws=0x90008) == 3
    assert call(n=0, weight=None, grad_weight=None, ws=None, nbytes=0) == 0
