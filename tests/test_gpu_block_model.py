"""A run of the operators together, as a training step and a serving step use them; graphs, streams."""

import pytest
import torch

import paper_2412_06355_amd as dendsn
from tests import seq_ref
from tests.parity import announce

pytestmark = pytest.mark.gpu


class Block:
    """norm(x + stream) -> delta rule -> norm(o + stream) -> cross entropy, q, k, v cut from the normed rows
    themselves (H K + H K + H V of D), gates from a leaf; every leaf's gradient; AdamW on all."""

    T, b, H, K, V, classes, io = 70, 3, 2, 16, 32, 50, "f32"

    def __init__(self, dev, state="f32"):
        gen = torch.Generator().manual_seed(1)
        self.D = 2 * self.H * self.K + self.H * self.V
        n = lambda *s: torch.randn(s, generator=gen).to(dev)
        self.rows = self.T * self.b
        self.x, self.stream = n(self.rows, self.D), n(self.rows, self.D)
        self.targets = torch.randint(0, self.classes, (self.rows,), generator=gen).to(dev)
        self.params = [1 + 0.1 * n(self.D), 1 + 0.1 * n(self.H * self.V), 0.2 * n(self.classes, self.H * self.V),
                       -0.3 * torch.rand((self.T, self.b, self.H), generator=gen).to(dev),
                       torch.rand((self.T, self.b, self.H), generator=gen).to(dev)]
        self.cfg = dendsn.DeltaRuleConfig(T=self.T, batch=self.b, H=self.H, K=self.K, V=self.V)
        self.n1 = dendsn.RMSNormConfig(N=self.rows, D=self.D)
        self.n2 = dendsn.RMSNormConfig(N=self.rows, D=self.H * self.V)
        self.ce = dendsn.LinearCEConfig(N=self.rows, V=self.classes, D=self.H * self.V)
        self.opt = dendsn.AdamWConfig(lr=1e-2, state=state)
        self.states = dendsn.adamw_states(self.opt, self.params)
        self.step_no = torch.ones((1,), dtype=torch.int32, device=dev)

    def cut(self, y):
        hk = self.H * self.K
        y = y.view(self.T, self.b, self.D)
        return (y[..., :hk].unflatten(-1, (self.H, self.K)), y[..., hk:2 * hk].unflatten(-1, (self.H, self.K)),
                y[..., 2 * hk:].unflatten(-1, (self.H, self.V)))

    def gradients(self):
        w1, w2, readout, g, beta = self.params
        y, rstd1, s1 = dendsn.rms_norm(self.n1, self.x, w1, self.stream)
        q, k, v = self.cut(y)
        k = k / self.K  # keys of norm 1 at most
        o, _, ckpt = dendsn.delta_rule(self.cfg, q, k, v, g, beta)
        z, rstd2, _ = dendsn.rms_norm(self.n2, o.view(self.rows, -1), w2)
        out = dendsn.linear_ce_train(self.ce, z, readout, self.targets)
        b2 = dendsn.rms_norm_backward(self.n2, o.view(self.rows, -1), w2, rstd2, out["grad_hidden"])
        back = dendsn.delta_rule_backward(self.cfg, q, k, v, g, beta, None, ckpt, b2["grad_x"].view(o.shape))
        gy = torch.cat([back["grad_q"].flatten(2), back["grad_k"].flatten(2) / self.K, back["grad_v"].flatten(2)], -1)
        b1 = dendsn.rms_norm_backward(self.n1, s1, w1, rstd1, gy.view(self.rows, self.D))
        return out["loss"], b1["grad_x"], [b1["grad_weight"], b2["grad_weight"], out["grad_weight"], back["grad_g"],
                                           back["grad_beta"]]

    def step(self):
        loss, grad_x, grads = self.gradients()
        dendsn.adamw(self.opt, self.params, grads, self.states, self.step_no, seed=3)
        self.step_no += 1
        return loss, grad_x

    def reference(self):
        """Loss and gradients by torch in float64, on the CPU."""
        leaves = [t.double().cpu().requires_grad_() for t in [self.x, *self.params]]
        x, w1, w2, readout, g, beta = leaves
        norm = lambda s, w: s / (s.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        q, k, v = self.cut(norm(x + self.stream.double().cpu(), w1))
        k = k / self.K
        S, o = torch.zeros((self.b, self.H, self.K, self.V), dtype=torch.float64), []
        for t in range(self.T):
            S = torch.exp(g[t])[..., None, None] * S
            u = beta[t][..., None] * (v[t] - (k[t][..., None] * S).sum(-2))
            S = S + k[t][..., None] * u[..., None, :]
            o.append(self.K ** -0.5 * (q[t][..., None] * S).sum(-2))
        z = norm(torch.stack(o).view(self.rows, -1), w2)
        logits = z @ readout.t()
        loss = torch.logsumexp(logits, 1) - logits.gather(1, self.targets.cpu()[:, None])[:, 0]
        grads = torch.autograd.grad(loss.sum(), leaves)
        return loss.detach(), grads[0], list(grads[1:])


def test_gradients_of_the_block(gpu_device):
    """Each operator is off by less than 1e-5 of its result (their own tests), in a chain of eight."""
    announce("block gradients")
    net = Block(gpu_device)
    loss, grad_x, grads = net.gradients()
    want, want_x, want_g = net.reference()
    for name, a, b in [("loss", loss, want), ("x", grad_x, want_x)] + [(str(i), *ab) for i, ab in enumerate(zip(grads, want_g))]:
        off = (a.double().cpu() - b).norm() / b.norm()
        assert off <= 8e-5, (name, float(off))


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_captured_step(gpu_device, state):
    """A training step captured in a graph, replayed with eager work between, against eager steps."""
    announce(f"block graph {state}")
    eager, net = Block(gpu_device, state), Block(gpu_device, state)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        warm = Block(gpu_device, state)
        warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grad_x = net.step()
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want, want_x = eager.step()
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(grad_x, want_x), i
        for a, b in zip(net.params, eager.params):
            assert torch.equal(a, b), i
        for a, b in zip(net.states, eager.states):
            for x, y in zip(a, b):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i


def test_two_streams(gpu_device):
    """The same step on two streams at once, each with workspaces of its own."""
    announce("block streams")
    want = Block(gpu_device).gradients()
    nets, got = [Block(gpu_device) for _ in range(2)], [None, None]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in nets]
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = nets[i].gradients()
    torch.cuda.synchronize()
    for loss, grad_x, grads in got:
        assert torch.equal(loss, want[0]) and torch.equal(grad_x, want[1])
        for a, b in zip(grads, want[2]):
            assert torch.equal(a, b)


def test_serving_step(gpu_device):
    """One token of three requests on slots, beside the same tokens in one call."""
    announce("block serving")
    net = Block(gpu_device)
    w1, w2, readout, g, beta = net.params
    y, _, _ = dendsn.rms_norm(net.n1, net.x, w1, net.stream)
    q, k, v = net.cut(y)
    k = k / net.K
    o, last, _ = dendsn.delta_rule(net.cfg, q, k, v, g, beta, save_ckpt=False)
    state = torch.zeros((5, net.H, net.K, net.V), device=gpu_device)
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device=gpu_device)
    one, step = net.n1.with_(N=net.b), net.cfg.with_(T=1)
    outs = []
    for t in range(net.T):
        at = slice(t * net.b, (t + 1) * net.b)
        row, _, _ = dendsn.rms_norm(one, net.x[at], w1, net.stream[at])
        assert torch.equal(row, y[at])
        hk = net.H * net.K
        qt, kt, vt = row[:, :hk].unflatten(-1, (net.H, -1)), row[:, hk:2 * hk].unflatten(-1, (net.H, -1)) / net.K, \
            row[:, 2 * hk:].unflatten(-1, (net.H, -1))
        outs.append(dendsn.delta_rule_step(step, qt, kt, vt, g[t], beta[t], state, slots))
    o2 = torch.stack(outs)
    assert (o2 - o).norm() <= 2e-5 * o.norm() and (state[slots.long()] - last).norm() <= 2e-5 * last.norm()
    assert not state[[1, 3]].any()
    s, _ = dendsn.linear_ce(net.ce, dendsn.rms_norm(net.n2, o2.view(net.rows, -1), w2)[0], readout, net.targets)
    assert torch.isfinite(s).all()
