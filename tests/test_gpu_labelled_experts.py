"""Cross entropy, rows in 8 bits and the layer of single steps together with the training operators: a step of
examples/labelled_experts.py against automatic differentiation in 64 bits, with rows in 8 bits against the same step over restored rows,
its answers, and all of it under a captured graph."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu

SIZES = [(40, 32, 48, 4, 2, 300), (75, 27, 33, 5, 3, 131), (1, 16, 16, 3, 1, 64), (300, 64, 96, 6, 2, 2000)]


def problem(tokens, width, hidden, experts, top_k, vocabulary, kept, dtype=torch.float32):
    from labelled_experts import Model
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, width), generator=g).to("cuda", dtype)
    label = torch.randint(0, vocabulary, (tokens,), generator=g)
    label[torch.rand(tokens, generator=g) < 0.2] = -100
    label[0] = 1
    weight = (0.5 + torch.rand(tokens, generator=g)).cuda()
    return Model(width, hidden, experts, top_k, vocabulary, seed=tokens, kept=kept, dtype=dtype), x, label.cuda(), weight


def plain_step(model, x, label, weight, balance):
    """Losses and gradients by automatic differentiation on the CPU; the routing is that of the logits."""
    p = {n: v.detach().double().cpu().requires_grad_() for n, v in model.p.items()}
    x = x.detach().double().cpu().requires_grad_()
    label, weight = label.cpu(), weight.double().cpu()
    experts, k = p["router"].shape[0], model.top_k
    z = x @ p["router"].T
    probability = torch.softmax(z, dim=1)
    chosen = torch.zeros_like(z).scatter_(1, torch.topk(z, k, dim=1)[1], 1.0)
    gate = probability * chosen
    gate = gate / gate.sum(1, keepdim=True)
    out = x
    for e in range(experts):
        h = torch.nn.functional.gelu(x @ p["w1"][e].T + p["b1"][e])
        out = out + gate[:, e:e + 1] * (h @ p["w2"][e].T + p["b2"][e])
    held = label >= 0
    log_q = torch.log_softmax(out @ p["head"].T, dim=1)
    loss = -torch.gather(log_q, 1, label.clamp(min=0)[:, None])[:, 0] * weight * held
    share = chosen.sum(0) / chosen.sum()
    (loss.sum() + balance * experts * (share.detach() * probability.sum(0)).sum() / x.shape[0]).backward()
    return loss.detach(), {**{n: v.grad for n, v in p.items()}, "x": x.grad}


@pytest.mark.parametrize("sizes", SIZES)
def test_a_step(sizes):
    """Gradients in 32 bits through eight operators: within 1e-4 of the largest of their array (sums of a few hundred to a few thousand
    terms of relative error 2^-24 each, passed through products with weights of norm about one)."""
    model, x, label, weight = problem(*sizes, kept=False)
    loss, gradients = model.step(x, label, weight=weight, balance=0.3)
    want_loss, want = plain_step(model, x, label, weight, 0.3)
    assert float((loss.cpu() - want_loss).abs().max()) <= 1e-4 * float(want_loss.abs().max())
    for name in ("w1", "b1", "w2", "b2", "router", "head", "x"):
        assert float((gradients[name].cpu() - want[name]).abs().max()) <= 1e-4 * float(want[name].abs().max()) + 1e-7, name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", SIZES)
def test_a_step_with_rows_in_8_bits(sizes, dtype):
    """The same losses as without, and the gradients of a way back over the restored rows, bit for bit."""
    model, x, label, weight = problem(*sizes, kept=True, dtype=dtype)
    loss, gradients = model.step(x, label, weight=weight, balance=0.3)
    plain, *_ = problem(*sizes, kept=False, dtype=dtype)
    plain_loss, _ = plain.step(x, label, weight=weight, balance=0.3)
    assert torch.equal(loss, plain_loss)
    out, (r, pre, *rows) = model.forward(x)
    lse = nb.nacho_xent(out, plain.p["head"], label, weight=weight)[1]
    g_out, _ = nb.nacho_xent_grad(out, plain.p["head"], label, lse, weight=weight, grad_head=False)
    restored = (r, nb.nacho_restore8(pre, dtype), *(nb.nacho_restore8(t, dtype) for t in rows))
    want = plain.backward(x @ plain.p["router"].T, g_out, restored, 0.3)
    for name, value in want.items():
        assert torch.equal(gradients[name], value), name


@pytest.mark.parametrize("tokens", [1, 7, 64])
def test_answers_are_those_of_the_trained_path(tokens):
    """One call and the operators one by one, in 32 bits: the same sums of at most 128 + 96 products in other orders (2^-14 of
    logits of size one)."""
    model, x, _, _ = problem(tokens, 64, 96, 6, 2, 300, kept=False)
    out, _ = model.forward(x)
    want = (out.double() @ model.p["head"].double().T.contiguous())
    assert float((model.answer(x).double() - want).abs().max()) <= 2.0 ** -14 * max(1.0, float(want.abs().max()))


def test_the_example_runs():
    from labelled_experts import train
    model, x, label, losses = train(steps=3)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses) and bool(model.answer(x[:5]).isfinite().all())


def test_under_a_captured_graph():
    """A whole step and an answer in two graphs, replayed in turn on other inputs with eager work between."""
    model, x, label, weight = problem(96, 64, 80, 6, 2, 900, kept=True)

    def work():
        loss, gradients = model.step(x, label, weight=weight)
        return [loss, *(gradients[n] for n in sorted(gradients)), model.answer(x[:9])]

    work()
    torch.cuda.synchronize()
    graphs, results = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            results.append(work())
    for seed in range(4):
        torch.manual_seed(seed)
        x.normal_()
        label.random_(-200, 900)
        graphs[0].replay()
        torch.cuda.synchronize()
        eager = work()
        graphs[1].replay()
        torch.cuda.synchronize()
        for result in results:
            assert all(torch.equal(a, b) for a, b in zip(result, eager))


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_whatever_the_default_type_is(default):
    model, x, label, weight = problem(40, 32, 48, 4, 2, 300, kept=True)

    def work():
        r = nb.nacho_route(x @ model.p["router"].T, 2)
        pre = nb.Kept8.empty(r.token.numel(), 48, x.device)
        h = nb.nacho_experts(x, model.p["w1"], r.expert_pos, token=r.token, act="gelu", pre=pre)
        loss, lse = nb.nacho_xent(x, model.p["head"], label, weight=weight)
        return [h, loss, lse, *nb.nacho_xent_grad(x, model.p["head"], label, lse), nb.nacho_restore8(nb.nacho_keep8(x)),
                *nb.nacho_experts_grad(h, nb.nacho_keep8(x), model.p["w1"], r.expert_pos, token=r.token, act="gelu", pre=pre), model.answer(x)]

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
    kept = nb.nacho_keep8(z)
    w = torch.zeros((1, 8, 8), device="cuda")
    label = torch.zeros(4, dtype=torch.int64, device="cuda")
    monkeypatch.setattr(nb, "_current_device", lambda: z.get_device() + 1)
    for call in (lambda: nb.nacho_xent(z, z, label), lambda: nb.nacho_keep8(z), lambda: nb.nacho_restore8(kept), lambda: nb.nacho_experts_step(z, z[:, :1], 1, w, w),
                 lambda: nb.nacho_experts_grad(z, kept, w, torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call()
