"""A small network on a stream of tokens, trained and served with the library's kernels.

Token rows hold input currents and leak gates side by side; the gated scan integrates the
currents over the sequence; a DendSN layer (Stateless Dendrite, P compartments on B branches)
sees each integrated state for T steps and answers with spikes, whose rates are read out over
the vocabulary:

    tokens -> embedding -> gated scan -> DendSN layer -> rates -> linear cross entropy

Training runs the same chain backward, operator by operator, with plain SGD.  Serving takes one
token of each request at a time: its row, one step of the scan on the request's state, the
layer, the scores.

    python examples/token_stream.py            # trains on a repeating text and continues it
"""

from __future__ import annotations

import os
import sys
from dataclasses import dataclass

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2412_06355_amd as dendsn  # noqa: E402


@dataclass(frozen=True)
class Shape:
    V: int = 64          # vocabulary
    C: int = 128         # neurons
    B: int = 2           # branches of a neuron
    k: int = 2           # compartments of a branch
    T: int = 4           # steps for which the layer sees a token's state
    length: int = 96     # tokens of a training sequence
    batch: int = 8
    io: str = "f32"

    @property
    def D(self) -> int:  # channels of the scan: one per compartment
        return self.C * self.B * self.k


class Network:
    def __init__(self, shape: Shape, device, seed: int = 0):
        s, g = shape, torch.Generator().manual_seed(seed)
        dt = torch.bfloat16 if s.io == "bf16" else torch.float32
        n = lambda *dims: torch.randn(dims, generator=g)
        rows = torch.cat([1.5 * n(s.V, s.D), 1.0 + n(s.V, s.D)], dim=1)  # currents, gates
        self.shape, self.device = s, device
        self.table = rows.to(dt).to(device)
        self.kappa = torch.rand((s.C, s.B), generator=g).to(device)
        self.readout = (n(s.V, s.C) * s.C ** -0.5).to(dt).to(device)
        self.scan = dendsn.GatedScanConfig(T=s.length, batch=s.batch, D=s.D, io=s.io)

    def layer(self, items: int) -> dendsn.DendSNConfig:
        s = self.shape
        return dendsn.DendSNConfig(T=s.T, batch=items, C=s.C, S=1, B=s.B, comps_per_branch=s.k, stateful=False,
                                   io=s.io, residual=True)

    def rows(self, tokens):
        """Currents and gates of the tokens (any shape), as two views of one lookup."""
        s = self.shape
        cfg = dendsn.EmbeddingConfig(n=tokens.numel(), V=s.V, D=2 * s.D, io=s.io)
        both = dendsn.embedding(cfg, tokens.reshape(-1), self.table).view(*tokens.shape, 2 * s.D)
        return both[..., :s.D], both[..., s.D:]

    def rates(self, states):
        """The layer's spike rates [items, C] for states [items, D], and what its backward needs."""
        s = self.shape
        items = states.shape[0]
        cfg = self.layer(items)
        x = states.reshape(1, items * s.C, s.B * s.k).expand(s.T, -1, -1).contiguous()
        spikes, _, ckpt = dendsn.forward(cfg, x, None, self.kappa)
        return spikes.view(s.T, items, s.C).float().mean(0).to(spikes.dtype), (cfg, x, ckpt)

    def train_step(self, tokens, lr: float) -> torch.Tensor:
        """One SGD step on tokens [length + 1, batch]; returns the mean loss (on the device)."""
        s = self.shape
        seen, wanted = tokens[:-1], tokens[1:].reshape(-1)
        x, g = self.rows(seen)
        h, _, ckpt = dendsn.gated_scan(self.scan, x, g)
        rates, (cfg, layer_x, layer_ckpt) = self.rates(h.view(-1, s.D))
        items = rates.shape[0]
        ce = dendsn.LinearCEConfig(N=items, V=s.V, D=s.C, io=s.io)
        weight = torch.full((items,), 1.0 / items, device=self.device)
        out = dendsn.linear_ce_train(ce, rates, self.readout, wanted, weight)
        # back: a rate is the mean of T spikes, a state is seen T times
        grad_spikes = (out["grad_hidden"].float() / s.T).to(rates.dtype).view(1, -1).expand(s.T, -1).contiguous()
        layer = dendsn.backward(cfg, layer_x, None, self.kappa, None, None, None, layer_ckpt, grad_spikes)
        grad_h = layer["grad_x"].float().sum(0).to(h.dtype).view(h.shape)
        back = dendsn.gated_scan_backward(self.scan, x, g, None, ckpt, grad_h)
        grad_rows = torch.cat([back["grad_x"], back["grad_g"]], dim=-1).view(items, 2 * s.D)
        emb = dendsn.EmbeddingConfig(n=items, V=s.V, D=2 * s.D, io=s.io)
        grad_table = dendsn.embedding_backward(emb, seen.reshape(-1), grad_rows)
        for param, grad in ((self.table, grad_table), (self.readout, out["grad_weight"]), (self.kappa, layer["grad_kappa"])):
            param.sub_(lr * grad)
        return out["loss"].mean()

    def serve(self, prompt, new: int):
        """Continues each request's prompt [length, batch] by ``new`` tokens, one at a time, each
        request on a state of its own; the likeliest token is taken (the lowest of equals)."""
        s, batch = self.shape, prompt.shape[1]
        state = torch.zeros((batch, s.D), device=self.device)
        slots = torch.arange(batch, device=self.device, dtype=torch.int32)
        step = self.scan.with_(T=1, batch=batch)
        out = []
        for t in range(prompt.shape[0] + new - 1):
            token = prompt[t] if t < prompt.shape[0] else out[-1]
            x, g = self.rows(token)
            h = dendsn.gated_scan_step(step, x, g, state, slots)
            if t >= prompt.shape[0] - 1:
                rates, _ = self.rates(h)
                out.append((rates.float() @ self.readout.float().t()).argmax(dim=1))
        return torch.stack(out)


def text(shape: Shape, rows: int, seed: int, device):
    """Sequences [rows, batch] that repeat a phrase of 12 tokens, each from a place of its own."""
    g = torch.Generator().manual_seed(seed)
    phrase = torch.randperm(shape.V, generator=g)[:12]
    start = torch.randint(0, 12, (shape.batch,), generator=g)
    return phrase[(torch.arange(rows)[:, None] + start) % 12].to(device)


def main():
    device = torch.device("cuda:0")
    shape = Shape()
    net = Network(shape, device)
    tokens = text(shape, shape.length + 1, 1, device)
    for i in range(60):
        loss = net.train_step(tokens, lr=1.0)
        if i % 10 == 9:
            print(f"step {i + 1}: loss {float(loss):.4f}", flush=True)
    prompt = tokens[:24]
    said = net.serve(prompt, 24)
    right = (said == tokens[24:48]).float().mean()
    print(f"continued 24 tokens of {shape.batch} requests, {100 * float(right):.0f} % as in the text", flush=True)


if __name__ == "__main__":
    main()
