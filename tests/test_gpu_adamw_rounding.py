"""8-bit optimizer states against another evaluation of the stated formulas, operation by operation in
fp32: the codes and the scales are the same, to the last bit.

Every operation that decides a rounding (products, sums, roots and quotients) is rounded to the
nearest on both sides, so nothing is allowed for.  A block's scale is its largest magnitude times 1/448
as fp32 has it, which is what torch makes of a division by 448 on the GPU; the quotient is another
number for half of all blocks.
"""

import numpy as np
import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests.parity import announce

pytestmark = pytest.mark.gpu

f32 = np.float32
BLOCK, TOP, PART, M32 = 256, f32(448), f32(1 / 448), 0xFFFFFFFF


def mix(h):
    """On arrays of uint64 that hold 32 bits."""
    for c in (0x7FEB352D, 0x9E3779B1, 0x846CA68B):
        h = ((h ^ (h >> np.uint64(16))) * np.uint64(c)) & np.uint64(M32)
    return h ^ (h >> np.uint64(16))


def bits_of(n, tensor, step, seed):
    u = lambda x: np.uint64(x & M32)
    key = mix(u(seed) ^ mix(u(seed >> 32) ^ mix(u(step) ^ mix(u(tensor + 1)))))
    i = np.arange(n, dtype=np.uint64)
    return mix(i ^ key)  # (places below 2^32)


def blocks(x):
    return np.pad(x, (0, -x.size % BLOCK)).reshape(-1, BLOCK)


def each(scales, n):
    return np.repeat(scales, BLOCK)[:n]


def rounded(x, u, positive):
    """(values in units of their block's scale, rounded by u in [0, 1), and the scales)"""
    top = np.abs(blocks(x)).max(axis=1)
    scale = np.where(top > 0, top * PART, f32(1)).astype(f32)
    size = np.minimum(np.abs(x) / each(scale, x.size), TOP)
    step = np.exp2(np.floor(np.log2(np.maximum(size, f32(2.0 ** -6)).astype(np.float64)))).astype(f32) / f32(8)
    code = np.floor(size / step + u) * step
    if positive:
        code = np.where(size > 0, np.maximum(code, f32(2.0 ** -9)), code)
    return np.copysign(code, x).astype(f32), scale


def step_of(held, g, b1, b2, bits):
    """New (m codes, m scales, root codes, root scales) from those held, as fp32 arrays."""
    m, ms, r, rs = held
    n = m.size
    m, r = m * each(ms, n), r * each(rs, n)
    m = f32(b1) * m + f32(1 - b1) * g
    v = f32(b2) * (r * r) + f32(1 - b2) * g * g
    u = [(x.astype(f32) * f32(2.0 ** -16)) for x in (bits & np.uint64(0xFFFF), bits >> np.uint64(16))]
    return (*rounded(m, u[0], False), *rounded(np.sqrt(v), u[1], True))


def codes(x):
    return torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seed", [3, (5 << 32) + 11])
def test_codes_and_scales_are_those_of_the_formulas(gpu_device, seed, grads):
    # more tensors than a launch has, some empty; a large one first and last
    sizes = [20001] + [(97 * i) % 1100 if i % 6 else 0 for i in range(48)] + [70000]
    gen = torch.Generator().manual_seed(seed % 1000)
    cfg = dendsn.AdamWConfig(beta1=0.9, beta2=0.99, state="e4m3")
    p = [0.05 * torch.randn((n,), generator=gen) for n in sizes]
    scale = torch.tensor([0.75])
    mine = [x.to(gpu_device) for x in p]
    states = dendsn.adamw_states(cfg, mine)
    held = [tuple(f32(1) * np.full(k, fill, f32) for k, fill in ((n, 0), (-(-n // BLOCK), 1)) * 2) for n in sizes]
    announce(f"adamw rounding {seed} {grads}")
    for step in (1, 2, 3, 1000):
        g = [(1e-2 * torch.randn((n,), generator=gen)).to(grads) for n in sizes]
        for x in g:
            x[::7] = 0      # values that a step brings nothing
        if step == 1:
            g[0][256:512] = 0  # a block of zeros
        dendsn.adamw(cfg, mine, [x.to(gpu_device) for x in g], states, step, grad_scale=scale.to(gpu_device), seed=seed)
        for i, n in enumerate(sizes):
            if n == 0:
                continue
            held[i] = step_of(held[i], g[i].float().numpy() * scale.numpy(), 0.9, 0.99, bits_of(n, i, step, seed))
            for name, got, want in zip(("m", "m scale", "root", "root scale"), states[i], held[i]):
                if got.dtype == torch.float8_e4m3fn:
                    got, want = got.view(torch.uint8).cpu(), codes(want)
                else:
                    got, want = got.cpu(), torch.from_numpy(want)
                off = got != want
                assert not bool(off.any()), f"{name} of tensor {i}, step {step}: {int(off.sum())} of {off.numel()} differ"


def test_a_scale_is_a_product():
    """And not the quotient: the two differ, so that the test above tells them apart."""
    top = np.exp(np.random.default_rng(0).uniform(-20, 5, 100000)).astype(f32)
    assert 0.4 < np.mean(top * PART != top / TOP) < 0.7 and f32(1) / f32(448) == PART
