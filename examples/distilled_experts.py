"""A small mixture of experts learns from the top logits of a teacher, through the library's training operators.

The student: a router, experts of two layers, the sum of the chosen experts' rows on top of the input, and a head over
the vocabulary.  One step runs

    routing (nacho_route)  ->  first and second layer (nacho_experts)  ->  sum (nacho_combine)  ->  loss against the
    teacher's stored logits, with the gradient of the student's (nacho_distill)

and the same back: nacho_combine_grad, nacho_experts_grad twice, nacho_combine for the rows of x that several slots read,
nacho_route_grad with the balance loss.  The router's and the head's products are plain matrix products.

    python examples/distilled_experts.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_17198_amd import binding as nb  # noqa: E402


class Student:
    def __init__(self, width, hidden, experts, top_k, vocabulary, seed=0, device="cuda", dtype=torch.float32):
        g = torch.Generator().manual_seed(seed)
        make = lambda *shape: (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(device, dtype)
        self.top_k = top_k
        self.p = dict(router=make(experts, width), w1=make(experts, hidden, width), b1=make(experts, hidden) * 0.1,
                      w2=make(experts, width, hidden), b2=make(experts, width) * 0.1, head=make(vocabulary, width))

    def step(self, x, teacher, temperature=1.0, balance=0.01, keep=None):
        """Losses of every token, the balance loss, and the gradients of the sum of the losses + `balance` times it.  Tokens
        that `keep` leaves out go past the experts."""
        p = self.p
        r = nb.nacho_route(x @ p["router"].T, self.top_k, normalise=True, keep=keep)
        pre = torch.empty((r.token.numel(), p["w1"].shape[1]), dtype=x.dtype, device=x.device)
        h = nb.nacho_experts(x, p["w1"], r.expert_pos, token=r.token, bias=p["b1"], act="gelu", pre=pre)
        y = nb.nacho_experts(h, p["w2"], r.expert_pos, bias=p["b2"])
        out = nb.nacho_combine(r.pos, r.slot, y, gate=r.gate, residual=x)
        logits = out @ p["head"].T
        g_logits = torch.empty_like(logits)
        loss, _ = nb.nacho_distill(teacher, logits, temperature=temperature, grad=g_logits)
        # back
        g = dict(head=g_logits.T @ out)
        g_out = g_logits @ p["head"]
        g_y, g_gate = nb.nacho_combine_grad(r.pos, r.slot, y, g_out, gate=r.gate)
        g["b2"], g["b1"] = torch.empty_like(p["b2"]), torch.empty_like(p["b1"])
        g_h, g["w2"] = nb.nacho_experts_grad(g_y, h, p["w2"], r.expert_pos, grad_bias=g["b2"])
        g_x, g["w1"] = nb.nacho_experts_grad(g_h, x, p["w1"], r.expert_pos, token=r.token, act="gelu", pre=pre, grad_bias=g["b1"])
        g_router = nb.nacho_route_grad(x @ p["router"].T, r, g_gate, balance=balance, keep=keep)
        g["router"] = g_router.T @ x
        # the input's: by way of the residual, the experts and the router
        g["x"] = nb.nacho_combine(r.pos, r.slot, g_x, residual=g_out) + g_router @ p["router"]
        return loss, r.balance, g

    def descend(self, gradients, rate):
        for name, value in self.p.items():
            value -= rate * gradients[name]


def top_logits(logits, keep):
    """The `keep` largest logits of every row as a CSR operand (columns ascending)."""
    rows, cols = logits.shape
    at = torch.sort(torch.topk(logits, keep, dim=1)[1], dim=1)[0]
    pos = torch.arange(rows + 1, dtype=torch.int32, device=logits.device) * keep
    return nb.csr(pos, at.to(torch.int32).reshape(-1), rows, cols, torch.gather(logits, 1, at).float().reshape(-1))


def train(steps=60, tokens=512, width=64, hidden=128, experts=8, top_k=2, vocabulary=1000, keep=32, rate=4.0, seed=0):
    """Mean loss of every step."""
    g = torch.Generator().manual_seed(seed + 1)
    x = torch.randn((tokens, width), generator=g).cuda()
    teacher = top_logits(3 * x @ torch.randn((width, vocabulary), generator=g).cuda() * width ** -0.5, keep)
    student = Student(width, hidden, experts, top_k, vocabulary, seed)
    losses = []
    for _ in range(steps):
        loss, balance, gradients = student.step(x, teacher)
        student.descend({name: value / tokens for name, value in gradients.items() if name != "x"}, rate)
        losses.append(loss.mean().item())
    return losses


if __name__ == "__main__":
    losses = train()
    print(f"mean loss {losses[0]:.4f} -> {losses[-1]:.4f}")
