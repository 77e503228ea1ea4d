"""Embedding rows and their gradient on the GPU against the definition."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


def make(n, V, D, io, kind, seed=0, index=torch.int64):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":          # a single id
        ids = torch.full((n,), V // 2)
    elif kind == "none":       # no token at all
        ids = torch.full((n,), -1)
    elif kind == "sorted":
        ids = torch.sort(torch.randint(0, V, (n,), generator=g)).values
    elif kind == "skewed":     # a few frequent ids, many rare ones, ids that are no row
        ids = (V * torch.rand((n,), generator=g) ** 4).long()
        ids = torch.where(torch.rand((n,), generator=g) < 0.1, torch.randint(-5, V + 5, (n,), generator=g), ids)
        if n > 2:
            ids[0], ids[1] = V, V - 1
            ids[2] = torch.iinfo(index).min
    else:
        ids = torch.randint(0, V, (n,), generator=g)
    dt = seq_ref.io_dtype(io)
    table = torch.randn((V, D), generator=g).to(dt)
    grad = torch.randn((n, D), generator=g).to(dt)
    return ids.to(index), table, grad


def forward_ref(ids, table, scale, V):
    ids = ids.long()
    keep = (ids >= 0) & (ids < V)
    rows = (table[ids.clamp(0, V - 1)].float() * scale).to(table.dtype)
    return torch.where(keep[:, None], rows, torch.zeros((), dtype=table.dtype))


CASES = [
    # n, V, D, kind: counts around a wave, a sorting block and a run of 64; tables around a pass's digit
    (1, 1, 1, "random"), (1, 5, 8, "none"), (2, 2, 3, "sorted"), (63, 7, 64, "skewed"), (64, 511, 65, "random"),
    (65, 512, 16, "one"), (127, 64, 8, "one"), (128, 33, 40, "one"), (129, 1, 24, "one"), (2047, 513, 8, "skewed"),
    (2048, 32, 128, "sorted"), (2049, 31, 513, "skewed"), (4500, 3, 8, "random"), (5000, 70000, 16, "skewed"),
    (9000, 262145, 8, "random"), (20000, 40, 72, "skewed"), (300, 5000, 1000, "random"), (3, 300, 520, "none")]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,D,kind", CASES)
def test_against_definition(gpu_device, n, V, D, kind, io):
    index = torch.int32 if n % 2 else torch.int64
    ids, table, grad = make(n, V, D, io, kind, seed=n, index=index)
    scale = 1.0 if D % 2 else 1.7
    cfg = dendsn.EmbeddingConfig(n=n, V=V, D=D, io=io, scale=scale)
    announce(f"embed {cfg} {kind} {index}")
    d = [t.to(gpu_device) for t in (ids, table, grad)]
    out = dendsn.embedding(cfg, d[0], d[1])
    got = dendsn.embedding_backward(cfg, d[0], d[2])
    again = dendsn.embedding_backward(cfg, d[0], d[2])
    scale32 = float(torch.tensor(scale, dtype=torch.float32))
    # one product, one rounding: bit for bit
    assert torch.equal(out.cpu(), forward_ref(ids, table, torch.tensor(scale, dtype=torch.float32), V))
    ref, bound = seq_ref.embed_backward(ids, grad, V, scale32, io)
    seq_ref.assert_within(got, ref, bound, "grad_table")
    named = torch.zeros(V, dtype=torch.bool)
    named[ids[(ids >= 0) & (ids < V)].long()] = True
    bits = got.cpu()[~named].view(torch.int16 if io == "bf16" else torch.int32)
    assert not bits.any(), "rows that no token names are +0"
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rows_that_lie_apart(gpu_device, io):
    """Table and gradient as slices of wider buffers (odd strides too), a gradient of one
    broadcast row, and NaN in rows that no token names."""
    n, V, D = 700, 50, 24
    ids, table, grad = make(n, V, D, io, "skewed", seed=3)
    cfg = dendsn.EmbeddingConfig(n=n, V=V, D=D, io=io)
    dev = [t.to(gpu_device) for t in (ids, table, grad)]
    want, want_grad = dendsn.embedding(cfg, dev[0], dev[1]), dendsn.embedding_backward(cfg, dev[0], dev[2])
    for pad, at in ((8, 0), (8, 8), (5, 3)):
        announce(f"embed strided {io} pad {pad} at {at}")
        wide_t = torch.full((V, D + pad), float("nan"), dtype=table.dtype, device=gpu_device)
        wide_g = torch.full((n, D + pad), float("nan"), dtype=table.dtype, device=gpu_device)
        wide_t[:, at:at + D], wide_g[:, at:at + D] = dev[1], dev[2]
        assert torch.equal(dendsn.embedding(cfg, dev[0], wide_t[:, at:at + D]), want)
        assert torch.equal(dendsn.embedding_backward(cfg, dev[0], wide_g[:, at:at + D]), want_grad)
    row = dev[2][:1].expand(n, D)
    assert torch.equal(dendsn.embedding_backward(cfg, dev[0], row), dendsn.embedding_backward(cfg, dev[0], row.contiguous()))
    holes = dev[2].clone()
    holes[(dev[0] < 0) | (dev[0] >= V)] = float("nan")
    assert torch.equal(dendsn.embedding_backward(cfg, dev[0], holes), want_grad)


def test_offsets_past_32_bits(gpu_device):
    """A table whose rows lie 2^26 elements apart (its last row starts past 2^32 bytes)."""
    V, D, n = 70, 64, 40
    store = torch.empty(((V - 1) << 26) + D, dtype=torch.bfloat16, device=gpu_device)
    table = store.as_strided((V, D), (1 << 26, 1))
    values = torch.randn((V, D)).bfloat16().to(gpu_device)
    table.copy_(values)
    ids = torch.arange(V - n, V, device=gpu_device)
    cfg = dendsn.EmbeddingConfig(n=n, V=V, D=D, io="bf16")
    announce(f"embed far rows {cfg}")
    assert torch.equal(dendsn.embedding(cfg, ids, table), values[ids])
    grad = store.as_strided((n, D), (1 << 26, 1))
    want = torch.zeros_like(values)
    want[ids] = values[:n]
    assert torch.equal(dendsn.embedding_backward(cfg, ids, grad), want)


def test_nothing(gpu_device):
    cfg = dendsn.EmbeddingConfig(n=0, V=6, D=5)
    ids = torch.zeros((0,), dtype=torch.int64, device=gpu_device)
    announce("embed n = 0")
    assert dendsn.embedding(cfg, ids, torch.ones((6, 5), device=gpu_device)).shape == (0, 5)
    got = dendsn.embedding_backward(cfg, ids, torch.zeros((0, 5), device=gpu_device))
    assert got.shape == (6, 5) and not got.view(torch.int32).any()
    none = dendsn.embedding(cfg.with_(n=3, V=0), torch.zeros(3, dtype=torch.int64, device=gpu_device),
                            torch.zeros((0, 5), device=gpu_device))
    assert none.shape == (3, 5) and not none.any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D", [3, 40])
def test_rows_without_a_token_are_plus_zero_at_any_scale(gpu_device, io, D):
    """The product of a negative scale with no sum would be -0."""
    n, V = 50, 70
    ids, _, grad = make(n, V, D, io, "random", seed=D)
    cfg = dendsn.EmbeddingConfig(n=n, V=V, D=D, io=io, scale=-2.0)
    announce(f"embed negative scale {cfg}")
    got = dendsn.embedding_backward(cfg, ids.to(gpu_device), grad.to(gpu_device))
    ref, bound = seq_ref.embed_backward(ids, grad, V, -2.0, io)
    seq_ref.assert_within(got, ref, bound, "grad_table")
    named = torch.zeros(V, dtype=torch.bool)
    named[ids] = True
    assert not named.all()
    assert not got.cpu()[~named].view(torch.int16 if io == "bf16" else torch.int32).any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,D", [(33000, 5000, 520), (40001, 300, 1025), (600001, 3000, 8), (1100000, 100, 3)])
def test_gradient_of_many_tokens(gpu_device, n, V, D, io):
    """Runs of 32 positions and their joins; sorting blocks of two and three rounds of 1024, whose
    bases are carried on."""
    ids, _, grad = make(n, V, D, io, "skewed", seed=n)
    cfg = dendsn.EmbeddingConfig(n=n, V=V, D=D, io=io, scale=0.5)
    announce(f"embed gradient {cfg}")
    d = [t.to(gpu_device) for t in (ids, grad)]
    got, again = (dendsn.embedding_backward(cfg, *d) for _ in range(2))
    ref, bound = seq_ref.embed_backward(ids, grad, V, 0.5, io)
    seq_ref.assert_within(got, ref, bound, "grad_table")
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))
