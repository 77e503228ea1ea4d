"""The bounds in norm of the delta rule's tests: the chunks' formulas are the recurrence's, and a term
left out, or operands of too few bits, exceed what the tests allow.  All on the CPU, in float64."""

import pytest
import torch

from tests import block_chunks, block_ref
from tests.test_gpu_delta import make
from tests.test_gpu_delta_norms import CASES, case_of


@pytest.mark.parametrize("T,b,H,Hk,K,V", [(1, 2, 2, 1, 3, 4), (64, 1, 2, 0, 8, 5), (130, 3, 4, 2, 12, 9)])
def test_chunks_are_the_recurrence(T, b, H, Hk, K, V):
    from paper_2412_06355_amd import DeltaRuleConfig

    cfg = DeltaRuleConfig(T=T, batch=b, H=H, Hk=Hk, K=K, V=V)
    for ragged, carry in ((False, False), (True, True)):
        d = make(cfg, T, ragged, carry)
        want = block_ref.delta(d, 0.7, "f32")
        got = block_chunks.delta(d, 0.7)
        for name, (value, _) in want.items():
            assert (got[name] - value).norm() <= 1e-12 * (1 + value.norm()), name


@pytest.mark.parametrize("case", CASES, ids=str)
def test_a_term_left_out_of_the_decays_gradient_shows(case):
    """Of every head of a sequence of more than one chunk, and ten times over of half of them.  Where a
    chunk's decays leave e^-9 of a state, its product ("held") is less than a rounding to bf16."""
    for io in ("f32", "bf16"):
        cfg, d, segments = case_of(case, io)
        ref = block_chunks.delta(d, cfg.K ** -0.5)
        bound = block_chunks.bounds(ref, cfg.K, io, segments)["grad_g"]
        long = torch.full((cfg.batch,), cfg.T) if d["lengths"] is None else d["lengths"].clamp(0, cfg.T)
        long = long > block_chunks.CHUNK
        assert bool(long.any())
        for name in block_chunks.TERMS:
            if name == "held" and io == "bf16" and case[7] > 0.2:
                continue
            without = block_chunks.delta(d, cfg.K ** -0.5, leave_out=(name,))
            over = (block_chunks.off(without["grad_g"], ref, "grad_g") / bound)[long]
            assert float(over.min()) > 1 and float(over.median()) > 10, (io, name, float(over.min()))


@pytest.mark.parametrize("case", CASES, ids=str)
def test_states_of_two_bf16_values_show(case):
    """Three bf16 values an operand are within the states' bound, two are not."""
    cfg, d, segments = case_of(case, "bf16")
    ref = block_chunks.delta(d, cfg.K ** -0.5)
    bound = block_chunks.bounds(ref, cfg.K, "bf16", segments)
    three, two = (block_chunks.delta(d, cfg.K ** -0.5, planes=n) for n in (3, 2))
    ran = torch.full((cfg.batch,), True) if d["lengths"] is None else d["lengths"] > block_chunks.CHUNK
    for name in ("s_last", "grad_s0"):
        assert bool((block_chunks.off(three[name], ref, name) <= bound[name]).all()), name
        away = block_chunks.off(two[name], ref, name)
        assert bool((away[ran] > bound[name][ran]).all()), (name, float((away / bound[name])[ran].min()))
