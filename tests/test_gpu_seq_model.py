"""The token-sequence operators as they are used together: training and serving of a small
network, on another stream than the default one, and captured in a HIP graph."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from examples.token_stream import Network, Shape, text
from tests.parity import announce

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_training_and_serving(gpu_device, io):
    """A repeating text is learnt (the loss of a uniform guess is log 64 = 4.2) and continued
    token by token; two runs from the same seed are the same, bit for bit."""
    shape = Shape(length=48, io=io)
    announce(f"token stream {shape}")
    tokens = text(shape, shape.length + 1, 1, gpu_device)
    runs = []
    for _ in range(2):
        net = Network(shape, gpu_device)
        losses = [net.train_step(tokens, lr=1.0) for _ in range(40)]
        runs.append((torch.stack(losses).cpu(), net))
    losses, net = runs[0]
    assert losses[-1] < 0.5 < losses[0]
    assert torch.equal(losses, runs[1][0]) and torch.equal(net.table, runs[1][1].table)
    said = net.serve(tokens[:24], 12)
    assert float((said == tokens[24:36]).float().mean()) > 0.9


def _inputs(device, seed, io):
    g = torch.Generator(device=device).manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    n = lambda *s: torch.randn(s, generator=g, device=device).to(dt)
    T, b, D, V = 200, 3, 48, 500
    d = dict(ids=torch.randint(-1, V, (T * b,), generator=g, device=device), table=n(V, 2 * D), readout=n(V, D),
             wanted=torch.randint(-1, V, (T * b,), generator=g, device=device),
             weight=torch.rand((T * b,), generator=g, device=device), state=torch.randn((b, D), generator=g, device=device))
    return (T, b, D, V), d


def _chain(dims, d, io):
    """Lookup, scan, loss, and all gradients; a serving step too."""
    T, b, D, V = dims
    emb = dendsn.EmbeddingConfig(n=T * b, V=V, D=2 * D, io=io)
    sc = dendsn.GatedScanConfig(T=T, batch=b, D=D, io=io)
    ce = dendsn.LinearCEConfig(N=T * b, V=V, D=D, io=io)
    rows = dendsn.embedding(emb, d["ids"], d["table"]).view(T, b, 2 * D)
    x, g = rows[..., :D], rows[..., D:]
    h, last, ckpt = dendsn.gated_scan(sc, x, g)
    out = dendsn.linear_ce_train(ce, h.view(-1, D), d["readout"], d["wanted"], d["weight"])
    out["alone"], _ = dendsn.linear_ce(ce, h.view(-1, D), d["readout"], d["wanted"])
    back = dendsn.gated_scan_backward(sc, x, g, None, ckpt, out["grad_hidden"].view(T, b, D))
    grad_rows = torch.cat([back["grad_x"], back["grad_g"]], dim=-1).view(T * b, 2 * D)
    out["grad_table"] = dendsn.embedding_backward(emb, d["ids"], grad_rows)
    state = d["state"].clone()
    out["stepped"] = dendsn.gated_scan_step(sc.with_(T=1), x[0], g[0], state)
    return dict(out, h=h, last=last, state=state)


def _same(a, b):
    for k in a:
        assert torch.equal(a[k].contiguous().view(torch.uint8), b[k].contiguous().view(torch.uint8)), k


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_another_stream(gpu_device, io):
    """The calls run on the current stream: inputs that a side stream writes just before are seen."""
    dims, d = _inputs(gpu_device, 3, io)
    announce(f"chain on a side stream {io}")
    want = _chain(dims, d, io)
    torch.cuda.synchronize(gpu_device)
    side = torch.cuda.Stream(device=gpu_device)
    late = {k: torch.zeros_like(v) for k, v in d.items()}
    side.wait_stream(torch.cuda.current_stream(gpu_device))
    with torch.cuda.stream(side):
        spin = torch.randn((4096, 4096), device=gpu_device)
        for _ in range(8):
            spin = spin @ spin * 1e-3
        for k in d:
            late[k].copy_(d[k])
        got = _chain(dims, late, io)
    side.synchronize()
    _same(got, want)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_graph_capture(gpu_device, io):
    """The whole chain captured once and replayed on other inputs, with eager work between the
    replays: every replay equals the eager call on the same inputs."""
    dims, d = _inputs(gpu_device, 5, io)
    announce(f"chain under graph capture {io}")
    side = torch.cuda.Stream(device=gpu_device)
    side.wait_stream(torch.cuda.current_stream(gpu_device))
    with torch.cuda.stream(side):
        _chain(dims, d, io)
    torch.cuda.current_stream(gpu_device).wait_stream(side)
    torch.cuda.synchronize(gpu_device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _chain(dims, d, io)
    torch.cuda.synchronize(gpu_device)
    for rep in range(3):
        _, fresh = _inputs(gpu_device, 6 + rep, io)
        for k in d:
            d[k].copy_(fresh[k])
        want = _chain(dims, fresh, io)
        for t in out.values():
            t.fill_(3)
        torch.cuda.synchronize(gpu_device)
        graph.replay()
        torch.cuda.synchronize(gpu_device)
        _same(out, want)
