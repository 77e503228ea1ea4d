"""The gated delta rule on the GPU in norm, head by head of every sequence, against the chunks' formulas in
float64: what bounds value by value are too wide for (the decay's gradient, the states of bf16
calls), and the scans' blocks of 32 columns over more chunks than they fetch ahead."""

import pytest

import paper_2412_06355_amd as dendsn
from tests import block_chunks
from tests.parity import announce
from tests.test_gpu_delta import make, run

# T, batch, H, Hk, K, V, whether lengths differ, largest decay, whether the steps go in segments
CASES = [
    (300, 2, 3, 1, 128, 48, False, 0.3, False),
    (200, 3, 2, 0, 60, 33, True, 0.05, False),
    # blocks of 32 columns, several a head, five and six chunks: all lengths around the chunks' ends
    (330, 8, 16, 8, 128, 64, True, 0.1, False),
    (330, 8, 16, 0, 69, 40, True, 0.1, False),
    (300, 8, 11, 0, 64, 96, True, 0.1, False),
    (300, 8, 16, 0, 21, 33, True, 0.1, False),
    # segments
    (1537, 3, 2, 1, 36, 33, True, 0.02, True),
    (2100, 1, 2, 0, 128, 64, False, 0.02, True),
]
LENGTHS = [0, 1, 65, 64, 129, 256, 320, 1 << 20]


def case_of(case, io):
    T, b, H, Hk, K, V, ragged, decay, segments = case
    cfg = dendsn.DeltaRuleConfig(T=T, batch=b, H=H, Hk=Hk, K=K, V=V, io=io)
    d = make(cfg, T + K, ragged, True, "fused", decay)
    if ragged and b == len(LENGTHS):
        d["lengths"] = d["lengths"].new_tensor(LENGTHS)
    elif ragged:
        d["lengths"][0] = T - 70
    return cfg, d, segments


@pytest.mark.gpu
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_norms(gpu_device, case, io):
    cfg, d, segments = case_of(case, io)
    announce(f"delta norms {cfg}")
    got = run(cfg, d, gpu_device)
    ref = block_chunks.delta(d, cfg.K ** -0.5)
    worst = {}
    for name, bound in block_chunks.bounds(ref, cfg.K, io, segments).items():
        away = block_chunks.off(got[name], ref, name)
        size = block_chunks.over_head(name, ref[name])
        worst[name] = (float((away / size.clamp_min(1e-30)).max()), float((away / bound).max()))
    print({k: f"{a:.2e} ({b:.2f} of its bound)" for k, (a, b) in worst.items()}, flush=True)
    assert all(b <= 1 for _, b in worst.values()), worst
