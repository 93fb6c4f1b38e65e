"""A small mixture of experts learns from labels with its activations kept in 8 bits, and answers token by token.

The model: a router, experts of two layers, the sum of the chosen experts' rows on top of the input, and a head over the
vocabulary.  A step of training runs

    routing (nacho_route)  ->  first layer, its rows kept in 8 bits (nacho_experts)  ->  second layer  ->  sum (nacho_combine)  ->
    cross entropy from the rows and the head, without logits (nacho_xent)

and the same back (nacho_xent_grad, nacho_combine_grad, nacho_experts_grad from the kept rows, nacho_route_grad); between the two it
holds the input and the layers' rows in 8 bits (nacho_keep8).  An answer takes the layer of experts in one call (nacho_experts_step).
The router's product, and the head's in an answer, are plain matrix products.

    python examples/labelled_experts.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_17198_amd import binding as nb  # noqa: E402


class Model:
    def __init__(self, width, hidden, experts, top_k, vocabulary, seed=0, device="cuda", dtype=torch.float32, kept=True):
        g = torch.Generator().manual_seed(seed)
        make = lambda *shape: (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(device, dtype)
        self.top_k, self.kept = top_k, kept
        self.p = dict(router=make(experts, width), w1=make(experts, hidden, width), b1=make(experts, hidden) * 0.1,
                      w2=make(experts, width, hidden), b2=make(experts, width) * 0.1, head=make(vocabulary, width))

    def forward(self, x):
        """The rows before the head, and what the way back needs."""
        p = self.p
        r = nb.nacho_route(x @ p["router"].T, self.top_k, normalise=True)
        slots, hidden = r.token.numel(), p["w1"].shape[1]
        pre = nb.Kept8.empty(slots, hidden, x.device) if self.kept else torch.empty((slots, hidden), dtype=x.dtype, device=x.device)
        h = nb.nacho_experts(x, p["w1"], r.expert_pos, token=r.token, bias=p["b1"], act="gelu", pre=pre)
        y = nb.nacho_experts(h, p["w2"], r.expert_pos, bias=p["b2"])
        out = nb.nacho_combine(r.pos, r.slot, y, gate=r.gate, residual=x)
        hold = nb.nacho_keep8 if self.kept else lambda t: t
        return out, (r, pre, hold(x), hold(h), hold(y))

    def backward(self, x_logits, g_out, kept, balance):
        """Gradients of the parameters and of the input."""
        p = self.p
        r, pre, x, h, y = kept
        rows = lambda t: nb.nacho_restore8(t, g_out.dtype) if self.kept else t
        g = dict(b1=torch.empty_like(p["b1"]), b2=torch.empty_like(p["b2"]))
        g_y, g_gate = nb.nacho_combine_grad(r.pos, r.slot, rows(y), g_out, gate=r.gate)
        g_h, g["w2"] = nb.nacho_experts_grad(g_y, h, p["w2"], r.expert_pos, grad_bias=g["b2"])
        g_x, g["w1"] = nb.nacho_experts_grad(g_h, x, p["w1"], r.expert_pos, token=r.token, act="gelu", pre=pre, grad_bias=g["b1"])
        g_router = nb.nacho_route_grad(x_logits, r, g_gate, balance=balance)
        g["router"] = g_router.T @ rows(x)
        g["x"] = nb.nacho_combine(r.pos, r.slot, g_x, residual=g_out) + g_router @ p["router"]
        return g

    def step(self, x, label, weight=None, balance=0.01):
        """Losses of every row (0 where the label is no word of the vocabulary), and the gradients of their sum + `balance` times the
        balance loss."""
        out, kept = self.forward(x)
        loss, lse = nb.nacho_xent(out, self.p["head"], label, weight=weight)
        g_out, g_head = nb.nacho_xent_grad(out, self.p["head"], label, lse, weight=weight)
        g = self.backward(x @ self.p["router"].T, g_out, kept, balance)
        g["head"] = g_head
        return loss, g

    def answer(self, x):
        """The logits of a few rows."""
        p = self.p
        out = nb.nacho_experts_step(x, x @ p["router"].T, self.top_k, p["w1"], p["w2"], up_bias=p["b1"], down_bias=p["b2"], act="gelu",
                                    normalise=True, residual=x)
        return out @ p["head"].T

    def descend(self, gradients, rate):
        for name, value in self.p.items():
            value -= rate * gradients[name]


def train(steps=60, tokens=512, width=64, hidden=128, experts=8, top_k=2, vocabulary=500, rate=4.0, seed=0):
    """The model, rows, their labels, and the mean loss of every step."""
    g = torch.Generator().manual_seed(seed + 1)
    x = torch.randn((tokens, width), generator=g).cuda()
    label = (x @ torch.randn((width, vocabulary), generator=g).cuda()).argmax(dim=1)
    model, losses = Model(width, hidden, experts, top_k, vocabulary, seed), []
    for _ in range(steps):
        loss, gradients = model.step(x, label)
        model.descend({name: value / tokens for name, value in gradients.items() if name != "x"}, rate)
        losses.append(loss.mean().item())
    return model, x, label, losses


if __name__ == "__main__":
    model, x, label, losses = train()
    right = sum(int((model.answer(x[i:i + 16]).argmax(dim=1) == label[i:i + 16]).sum()) for i in range(0, 64, 16))
    print(f"mean loss {losses[0]:.4f} -> {losses[-1]:.4f}; {right} of 64 answers right")
