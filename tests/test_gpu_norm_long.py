"""The norm over more long rows than one launch has, of an x whose rows overlap: 2^23 and some rows of
8200 values in 8 bits are 64 GiB, their x is 16 MiB."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import block_ref, seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


def test_many_long_rows(gpu_device):
    n, D = (1 << 23) + 3, 8200  # 2^21 rows a launch
    gen = torch.Generator().manual_seed(1)
    flat = torch.randn((n + D - 1,), generator=gen).bfloat16().to(gpu_device)
    x = flat.as_strided((n, D), (1, 1))
    w = (1 + 0.1 * torch.randn((D,), generator=gen)).bfloat16().to(gpu_device)
    cfg = dendsn.RMSNormConfig(N=n, D=D, io="bf16")
    some = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 22) + 5, 3 << 21, (1 << 23) - 1, 1 << 23, n - 1], device=gpu_device)
    announce("norm of many long rows, e4m3")
    y, scale, rstd, summed = dendsn.rms_norm_e4m3(cfg, x, w)
    assert summed is None
    few = torch.stack([flat[i:i + D] for i in some.tolist()])
    want = dendsn.rms_norm_e4m3(cfg.with_(N=len(some)), few, w)
    for got, alone in zip((y.view(torch.uint8), scale, rstd), (want[0].view(torch.uint8), *want[1:3])):
        assert torch.equal(got[some], alone)
    value, bound = block_ref.norm(few, w, None, 1e-6, "bf16")["rstd"]
    seq_ref.assert_within(rstd[some], value, bound, "rstd")
