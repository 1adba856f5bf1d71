"""Federated distillation of a small language model, on one GPU: clients' local steps, their compressed updates, the server.

The model says the next token from the last one: its embedding (scaled), a layer norm, and the logits against the same
table.  A teacher has published its top logits for every client's texts.  Each round a client computes its loss and all its
gradients, which the operators leave in one flat fp32 vector; the vector is sent as a variable-length stream (two of a
hundred coordinates, 10 and 8 bits each), and the server adds the clients' decoded updates to the model.

    python examples/local_step.py [--rounds 20] [--clients 4]
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
    """A flat fp32 vector and its parts: the table (vocab, dim), gamma and beta of the norm."""

    def __init__(self, vocab: int, dim: int, device: str):
        self.vocab, self.dim = vocab, dim
        self.flat = torch.empty(vocab * dim + 2 * dim, device=device)
        self.table, self.gamma, self.beta = self.parts(self.flat)

    def parts(self, flat: torch.Tensor):
        end = self.vocab * self.dim
        return flat[:end].view(self.vocab, self.dim), flat[end:end + self.dim], flat[end + self.dim:]


class Client:
    """Texts of n tokens, the teacher's lists for them, and every buffer of a local step."""

    def __init__(self, model: Model, ids: torch.Tensor, teacher_ids: torch.Tensor, teacher_values: torch.Tensor, temperature: float):
        n, vocab, dim, dev = ids.numel(), model.vocab, model.dim, ids.device
        self.model, self.ids, self.teacher, self.T = model, ids, (teacher_ids, teacher_values), temperature
        there = ids >= 0                                                          # padding carries no loss
        self.weights = there.float() / there.sum()
        self.x, self.y, self.dy = (torch.empty(n, dim, device=dev) for _ in range(3))
        self.stats, self.logits, self.loss = torch.empty(n, 2, device=dev), torch.empty(n, vocab, device=dev), torch.empty(n, device=dev)
        self.update = torch.empty_like(model.flat)
        self.ws_table = cv.new_workspace(cv.embed_grad_workspace_bytes(n, vocab, dim), dev)
        self.ws_norm = cv.new_workspace(cv.layer_norm_grad_workspace_bytes(n, dim), dev)
        self.ws_loss = cv.new_workspace(cv.distill_workspace_bytes(n, vocab), dev)

    def step(self, rate: float) -> torch.Tensor:
        """The local step: `update` becomes -rate times the gradient.  Returns the mean loss (on the device)."""
        m, scale = self.model, math.sqrt(self.model.dim)
        dtable, dgamma, dbeta = m.parts(self.update)
        cv.embed(self.ids, m.table, self.x, scale=scale)
        cv.layer_norm(self.x, m.gamma, m.beta, self.y, self.stats)
        torch.mm(self.y, m.table.t(), out=self.logits)
        cv.distill(self.logits, *self.teacher, self.loss, self.ws_loss, temperature=self.T, weights=self.weights, dlogits=self.logits)
        torch.mm(self.logits, m.table, out=self.dy)
        torch.mm(self.logits.t(), self.y, out=dtable)                             # the table as it makes the logits ...
        cv.layer_norm_grad(self.dy, self.x, self.stats, m.gamma, self.dy, dgamma, dbeta, self.ws_norm)
        cv.embed_grad(self.ids, self.dy, dtable, self.ws_table, scale=scale, accumulate=True)   # ... and as it is looked up
        self.update.mul_(-rate)
        return self.loss.sum()


def run(rounds: int = 20, clients: int = 4, n: int = 512, vocab: int = 2000, dim: int = 64, k: int = 16, rate: float = 4.0,
        temperature: float = 2.0, seed: int = 1, device: str = "cuda:0", say=print):
    """Returns the rounds' mean losses."""
    g = torch.Generator(device=device).manual_seed(seed)
    model = Model(vocab, dim, device)
    model.table.normal_(0.0, dim ** -0.5, generator=g)
    model.gamma.fill_(1.0)
    model.beta.zero_()
    follows = torch.randint(vocab, (vocab, k), device=device, generator=g)       # what the teacher expects after each token
    group = []
    for _ in range(clients):
        ids = torch.randint(vocab // 4, (n,), device=device, generator=g)
        ids[-n // 8:] = -1
        values = 8.0 - torch.arange(k, device=device) * 0.5
        group.append(Client(model, ids, follows[ids.clamp(min=0)], values.expand(n, k).contiguous(), temperature))
    d = model.flat.numel()
    plan = cv.plan(d, code_len=(10, 8), fractions=(0.005, 0.015))
    streams = [cv.new_stream_buffer(plan, device) for _ in group]
    ws_encode = cv.new_workspace(cv.encode_workspace_bytes(d, clients), device)
    ws_decode = cv.new_workspace(cv.decode_workspace_bytes(d, clients), device)
    total, losses = torch.empty(d, device=device), []
    for turn in range(rounds):
        loss = torch.stack([c.step(rate) for c in group]).mean()
        cv.encode_batch([plan] * clients, [c.update for c in group], seed + turn, list(range(clients)), streams, ws_encode)
        cv.decode_aggregate(streams, total, ws_decode)
        model.flat.add_(total, alpha=1.0 / clients)
        losses.append(loss.item())
        bad = [cv.device_status(ws) for ws in (ws_encode, ws_decode, *(c.ws_table for c in group))]
        if any(bad):
            raise RuntimeError(f"device status {bad}")
        say(f"round {turn}: loss {losses[-1]:.4f}, {plan.total_bits / d:.3f} bits a coordinate")
    return losses


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--rounds", type=int, default=20)
    p.add_argument("--clients", type=int, default=4)
    a = p.parse_args()
    run(a.rounds, a.clients)
