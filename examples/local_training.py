"""Federated training of a small recurrent language model, on one GPU: clients' own AdamW steps, their compressed updates, the
server, and text from the model they have made.

The model is one gated layer: a token's embedding (scaled), a layer norm, two products that make its input and its gate,
the gated scan over its text, and the logits of the next token against the same table.  Each round a client takes the
server's weights, trains on its texts for some steps of AdamW with its averages in 8 bits, and sends the difference as a
variable-length stream (two of a hundred coordinates, 10 and 8 bits each); the server adds the decoded updates up.

    python examples/local_training.py [--rounds 10] [--clients 4]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2402_03770_amd.cvlc as cv  # noqa: E402


class Model:
    """A flat fp32 vector and its parts: the table (vocab, dim), the input's and the gate's matrix, gamma and beta of the norm."""

    def __init__(self, vocab: int, dim: int, device: str):
        self.vocab, self.dim = vocab, dim
        self.flat = torch.empty(vocab * dim + 2 * dim * dim + 2 * dim, device=device)
        self.table, self.input, self.gate, self.gamma, self.beta = self.parts(self.flat)

    def parts(self, flat: torch.Tensor):
        v, d = self.vocab, self.dim
        table, inp, gate, gamma, beta = flat.split([v * d, d * d, d * d, d, d])
        return table.view(v, d), inp.view(d, d), gate.view(d, d), gamma, beta


class Client:
    """Texts one after the other (text i's tokens are ids[starts[i]:starts[i + 1]], negative ones padding), a copy of the
    model, AdamW's averages and every buffer of a step."""

    def __init__(self, server: Model, ids: torch.Tensor, starts: torch.Tensor, decay: float = 0.01):
        n, vocab, dim, dev = ids.numel(), server.vocab, server.dim, ids.device
        self.server, self.model, self.ids, self.starts, self.taken = server, Model(vocab, dim, dev), ids, starts, 0
        self.labels = torch.full_like(ids, -1)                                    # the next token, but for a text's last
        self.labels[:-1] = ids[1:]
        self.labels[starts[1:].long() - 1] = -1
        self.labels[ids < 0] = -1
        there = self.labels >= 0
        self.weights = there.float() / there.sum()
        self.x, self.y, self.u, self.f, self.h, self.dh, self.du, self.df, self.dy = (torch.empty(n, dim, device=dev) for _ in range(9))
        self.norm_stats, self.stats, self.loss = torch.empty(n, 2, device=dev), torch.empty(n, 2, device=dev), torch.empty(n, device=dev)
        self.grad, self.update = torch.empty_like(server.flat), torch.empty_like(server.flat)
        self.m, self.v = (torch.zeros(server.flat.numel(), dtype=torch.uint8, device=dev) for _ in range(2))
        params, grads, ms, vs = (self.model.parts(t) for t in (self.model.flat, self.grad, self.m, self.v))
        scales = [torch.zeros(-(-p.numel() // cv.ADAMW_BLOCK), 2, device=dev) for p in params]
        self.plan = cv.AdamwPlan(params, grads, ms, vs, scales=scales, weight_decays=[decay] * 3 + [0.0] * 2,
                                 m_by_chance=True)
        self.ws_table = cv.new_workspace(cv.embed_grad_workspace_bytes(n, vocab, dim), dev)
        self.ws_norm = cv.new_workspace(cv.layer_norm_grad_workspace_bytes(n, dim), dev)
        self.ws_scan = cv.new_workspace(cv.gated_scan_workspace_bytes(n, dim, starts.numel() - 1), dev)
        self.ws_loss = cv.new_workspace(max(cv.linear_xent_workspace_bytes(n, vocab, dim, torch.float32),
                                            cv.linear_xent_grad_workspace_bytes(n, vocab, dim, torch.float32)), dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def gradient(self) -> torch.Tensor:
        """`grad` becomes the gradient of the mean loss, which is returned (on the device)."""
        m, scale = self.model, math.sqrt(self.model.dim)
        dtable, dinput, dgate, dgamma, dbeta = m.parts(self.grad)
        cv.embed(self.ids, m.table, self.x, scale=scale, status=self.status)
        cv.layer_norm(self.x, m.gamma, m.beta, self.y, self.norm_stats)
        torch.mm(self.y, m.input, out=self.u)
        torch.mm(self.y, m.gate, out=self.f)
        cv.gated_scan(self.u, self.f, self.h, self.ws_scan, starts=self.starts, status=self.status)
        cv.linear_xent(self.h, m.table, self.labels, self.loss, self.ws_loss, weights=self.weights, stats_out=self.stats, status=self.status)
        cv.linear_xent_grad(self.h, m.table, self.labels, self.stats, self.dh, dtable, self.ws_loss, weights=self.weights)
        cv.gated_scan_grad(self.dh, self.u, self.f, self.h, self.du, self.df, self.ws_scan, starts=self.starts)
        torch.mm(self.y.t(), self.du, out=dinput)
        torch.mm(self.y.t(), self.df, out=dgate)
        torch.mm(self.du, m.input.t(), out=self.dy)
        self.dy.addmm_(self.df, m.gate.t())
        cv.layer_norm_grad(self.dy, self.x, self.norm_stats, m.gamma, self.dy, dgamma, dbeta, self.ws_norm)
        cv.embed_grad(self.ids, self.dy, dtable, self.ws_table, scale=scale, accumulate=True)    # beside what the logits gave
        return self.loss.sum()

    def train(self, steps: int, rate: float, seed: int) -> torch.Tensor:
        """From the server's weights, `steps` steps; `update` becomes what they changed.  Returns the first step's loss."""
        self.model.flat.copy_(self.server.flat)
        first = None
        for _ in range(steps):
            loss = self.gradient()
            first = loss if first is None else first
            self.taken += 1
            cv.adamw(self.plan, self.taken, rate, seed=seed, status=self.status)
        torch.sub(self.model.flat, self.server.flat, out=self.update)
        return first


def write(model: Model, first: torch.Tensor, length: int) -> torch.Tensor:
    """(length, n) tokens that the model has most faith in after `first` (n), one token of every text at a time."""
    n, dim, dev = first.numel(), model.dim, first.device
    x, y, h, states = torch.empty(n, dim, device=dev), torch.empty(n, dim, device=dev), torch.empty(n, dim, device=dev), torch.zeros(n, dim, device=dev)
    out, now = [], first
    for _ in range(length):
        cv.embed(now, model.table, x, scale=math.sqrt(dim))
        cv.layer_norm(x, model.gamma, model.beta, y)
        cv.gated_scan_step(y @ model.input, y @ model.gate, states, h)
        now = (h @ model.table.t()).argmax(1)
        out.append(now)
    return torch.stack(out)


def run(rounds: int = 10, clients: int = 4, steps: int = 5, texts: int = 16, length: int = 64, vocab: int = 2000, dim: int = 64,
        rate: float = 3e-3, seed: int = 1, device: str = "cuda:0", say=print):
    """Returns the rounds' mean losses and some text of the last model."""
    g = torch.Generator(device=device).manual_seed(seed)
    server = Model(vocab, dim, device)
    server.flat.normal_(0.0, dim ** -0.5, generator=g)
    server.gamma.fill_(1.0)
    server.beta.zero_()
    follows = torch.randint(vocab // 4, (vocab,), device=device, generator=g)    # the language: a token, and what comes after it
    group = []
    for _ in range(clients):
        ids = torch.empty(texts, length, dtype=torch.int64, device=device)
        ids[:, 0] = torch.randint(vocab // 4, (texts,), device=device, generator=g)
        for t in range(1, length):
            ids[:, t] = follows[ids[:, t - 1]]
        starts = torch.arange(texts + 1, dtype=torch.int32, device=device) * length
        group.append(Client(server, ids.view(-1), starts))
    d = server.flat.numel()
    plan = cv.plan(d, code_len=(10, 8), fractions=(0.005, 0.015))
    streams = [cv.new_stream_buffer(plan, device) for _ in group]
    ws_encode = cv.new_workspace(cv.encode_workspace_bytes(d, clients), device)
    ws_decode = cv.new_workspace(cv.decode_workspace_bytes(d, clients), device)
    total, losses = torch.empty(d, device=device), []
    for turn in range(rounds):
        loss = torch.stack([c.train(steps, rate, seed + i) for i, c in enumerate(group)]).mean()
        cv.encode_batch([plan] * clients, [c.update for c in group], seed + turn, list(range(clients)), streams, ws_encode)
        cv.decode_aggregate(streams, total, ws_decode)
        server.flat.add_(total, alpha=1.0 / clients)
        losses.append(loss.item())
        bad = [cv.device_status(ws) for ws in (ws_encode, ws_decode, *(c.ws_table for c in group))] + [c.status.item() for c in group]
        if any(bad):
            raise RuntimeError(f"device status {bad}")
        say(f"round {turn}: loss {losses[-1]:.4f}, {plan.total_bits / d:.3f} bits a coordinate")
    return losses, write(server, group[0].ids[:4].clone(), 8)


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--rounds", type=int, default=10)
    p.add_argument("--clients", type=int, default=4)
    a = p.parse_args()
    run(a.rounds, a.clients)
