"""The training operators together: a step of examples/distilled_experts.py against automatic differentiation in 64 bits,
with strided operands and masked tokens, under a captured graph, and over some steps of training."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu


def plain_step(student, x, teacher, temperature, balance, keep):
    """Losses, balance loss and gradients by automatic differentiation on the CPU; the routing is that of the logits."""
    p = {n: v.detach().double().cpu().requires_grad_() for n, v in student.p.items()}
    x = x.detach().double().cpu().requires_grad_()
    tokens, experts, k = x.shape[0], p["router"].shape[0], student.top_k
    z = x @ p["router"].T
    probability = torch.softmax(z, dim=1)
    chosen = torch.zeros_like(z).scatter_(1, torch.topk(z, k, dim=1)[1], 1.0) * keep.double()[:, None]
    gate = probability * chosen
    gate = gate / gate.sum(1, keepdim=True).clamp(min=1e-300)
    out = x
    for e in range(experts):
        h = torch.nn.functional.gelu(x @ p["w1"][e].T + p["b1"][e])
        out = out + gate[:, e:e + 1] * (h @ p["w2"][e].T + p["b2"][e])
    logits = out @ p["head"].T / temperature
    pos, crd = teacher.keep[0].tolist(), teacher.keep[1].long().cpu()
    u = torch.full_like(logits, -math.inf)
    for t in range(tokens):
        u[t, crd[pos[t]:pos[t + 1]]] = teacher.val[pos[t]:pos[t + 1]].double().cpu() / temperature
    log_p = torch.log_softmax(u, dim=1)
    log_q = torch.log_softmax(logits, dim=1)
    weight = torch.exp(log_p)
    loss = torch.where(weight > 0, weight * (log_p - log_q), torch.zeros_like(weight)).sum(1) * temperature ** 2
    share = chosen.sum(0) / chosen.sum()
    even = experts * (share.detach() * (probability * keep.double()[:, None]).sum(0)).sum() / keep.sum()
    (loss.sum() + balance * even).backward()
    return loss.detach(), even.detach(), {**{n: v.grad for n, v in p.items()}, "x": x.grad}


@pytest.mark.parametrize("tokens,width,hidden,experts,top_k,vocabulary", [(40, 32, 48, 4, 2, 300), (75, 27, 33, 5, 3, 131), (1, 16, 16, 3, 1, 64)])
@pytest.mark.parametrize("masked", [False, True])
def test_a_step(tokens, width, hidden, experts, top_k, vocabulary, masked):
    """Gradients in 32 bits through seven operators: within 1e-4 of the largest of their array (sums of a few hundred terms of
    relative error 2^-24 each, passed through products with weights of norm about one)."""
    from distilled_experts import Student, top_logits
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, width), generator=g).cuda()
    keep = (torch.rand(tokens, generator=g) < 0.8) if masked and tokens > 1 else torch.ones(tokens, dtype=torch.bool)
    student = Student(width, hidden, experts, top_k, vocabulary, seed=tokens)
    teacher = top_logits(torch.randn((tokens, vocabulary), generator=g).cuda() * 2, 12)
    loss, even, gradients = student.step(x, teacher, temperature=1.5, balance=0.3, keep=keep.cuda() if masked else None)
    want_loss, want_even, want = plain_step(student, x, teacher, 1.5, 0.3, keep)
    assert float((loss.cpu() - want_loss).abs().max()) <= 1e-4 * float(want_loss.abs().max())
    assert abs(even.item() - want_even.item()) <= 1e-5 * want_even.item()
    for name, value in want.items():
        if name in ("w1", "b1", "w2", "b2", "router", "head", "x"):
            assert float((gradients[name].cpu() - value).abs().max()) <= 1e-4 * float(value.abs().max()) + 1e-7, name


def test_training_lowers_the_loss():
    from distilled_experts import train
    losses = train(steps=25)
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.7 * losses[0]


def test_under_a_captured_graph():
    """Every operator in a graph that is replayed on other inputs, with eager work between the replays."""
    tokens, experts, k, width, outer, vocabulary = 96, 6, 2, 64, 72, 9000
    new = lambda *shape: torch.randn(shape, device="cuda")
    z, x, w, gy, go, logits = new(tokens, experts), new(tokens, width), new(experts, outer, width), new(tokens * k, outer), new(tokens, outer), new(tokens, vocabulary)
    gate = torch.rand(tokens * k, device="cuda")
    pos = torch.arange(tokens + 1, dtype=torch.int32, device="cuda") * 5
    crd = (torch.arange(tokens * 5, device="cuda") % 5 * 1700 + 3).to(torch.int32)
    teacher = nb.csr(pos, crd, tokens, vocabulary, new(tokens * 5))
    few = nb.csr(pos[:3].contiguous(), crd[:10].contiguous(), 2, vocabulary * 8, teacher.val[:10])
    wide = new(2, vocabulary * 8)

    def work():
        r = nb.nacho_route(z, k)
        pre = torch.zeros((tokens * k, outer), device="cuda")
        y = nb.nacho_experts(x, w, r.expert_pos, token=r.token, act="silu", pre=pre)
        bias = torch.zeros((experts, outer), device="cuda")
        out = [r.expert, r.slot, r.gate, r.token, r.counts, r.lse, r.balance, y, pre, nb.nacho_combine(r.pos, r.slot, y, gate=r.gate),
               *nb.nacho_combine_grad(r.pos, r.slot, y, go, gate=r.gate), nb.nacho_route_grad(z, r, gate, balance=0.5),
               *nb.nacho_experts_grad(gy, x, w, r.expert_pos, token=r.token, act="silu", pre=pre, grad_bias=bias), bias]
        grad, more = torch.zeros_like(logits), torch.zeros_like(wide)
        loss, lse = nb.nacho_distill(teacher, logits, grad=grad)
        out += [loss, lse, grad, nb.nacho_distill_grad(teacher, logits, lse), *nb.nacho_distill(few, wide, grad=more), more, *nb.nacho_distill(few, wide)]
        return out

    for _ in range(2):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    for seed in range(4):
        torch.manual_seed(seed)
        for t in (z, x, w, gy, go, logits, wide):
            t.normal_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, work()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_whatever_the_default_type_is(default):
    """The operators' results under another default type of torch, bit for bit."""
    new = lambda *shape: torch.randn(shape, device="cuda", dtype=torch.float32)
    z, x, w, logits = new(40, 6), new(40, 32), new(6, 24, 32), new(40, 300)
    pos = torch.arange(41, dtype=torch.int32, device="cuda") * 5
    crd = (torch.arange(200, device="cuda") % 5 * 50).to(torch.int32)
    teacher = nb.csr(pos, crd, 40, 300, new(200))

    def work():
        r = nb.nacho_route(z, 2)
        y = nb.nacho_experts(x, w, r.expert_pos, token=r.token)
        loss, lse = nb.nacho_distill(teacher, logits)
        return [r.gate, r.lse, r.balance, y, nb.nacho_combine(r.pos, r.slot, y, gate=r.gate), *nb.nacho_combine_grad(r.pos, r.slot, y, x[:, :24], gate=r.gate),
                nb.nacho_route_grad(z, r, r.gate, balance=0.5), *nb.nacho_experts_grad(y, x, w, r.expert_pos, token=r.token), loss, lse,
                nb.nacho_distill_grad(teacher, logits, lse)]

    first, before = work(), torch.get_default_dtype()
    try:
        torch.set_default_dtype(default)
        second = work()
    finally:
        torch.set_default_dtype(before)
    for a, b in zip(first, second):
        assert a.dtype is torch.float32 and torch.equal(a, b)


def test_rows_of_another_gpu_are_refused(monkeypatch):
    """Kernels go to the current GPU's stream; rows have to be there."""
    z = torch.zeros((4, 8), device="cuda")
    monkeypatch.setattr(nb, "_current_device", lambda: z.get_device() + 1)
    for call in (lambda: nb.nacho_route(z, 2), lambda: nb.nacho_experts(z, torch.zeros((1, 8, 8), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")),
                 lambda: nb.nacho_combine(torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), z)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradients_that_are_not_wanted(act):
    """The others are the same bits, whichever are left out."""
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    bounds = torch.tensor([0, 30, 30, 77], dtype=torch.int32, device="cuda")
    x, w, gy, pre = new(77, 48), new(3, 40, 48), new(77, 40), new(77, 40)

    def run(wanted):
        bias = new(3, 40) if wanted[2] else None
        gx, gw = nb.nacho_experts_grad(gy, x, w, bounds, act=act, pre=pre, grad_x=None if wanted[0] else False,
                                       grad_weight=None if wanted[1] else False, grad_bias=bias)
        return gx, gw, bias

    every = run((True, True, True))
    for number in range(8):
        wanted = tuple(bool(number >> i & 1) for i in range(3))
        for got, want, asked in zip(run(wanted), every, wanted):
            assert torch.equal(got, want) if asked else got is None
    pos, slot = torch.tensor([0, 2, 2, 4], dtype=torch.int32, device="cuda"), torch.tensor([0, 3, 1, 2], dtype=torch.int32, device="cuda")
    y, go, gate = new(4, 33), new(3, 33), new(4)
    both = nb.nacho_combine_grad(pos, slot, y, go, gate=gate)
    only, none = nb.nacho_combine_grad(pos, slot, y, go, gate=gate, grad_gate=False)
    assert torch.equal(only, both[0]) and none is None
    none, only = nb.nacho_combine_grad(pos, slot, y, go, gate=gate, grad_y=False)
    assert torch.equal(only, both[1]) and none is None
