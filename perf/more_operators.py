"""Operators of a mixture-of-experts language model, as timed cases: its loss, its kept activations, its single steps.

Three operators beside those of a training step.  The cross entropy of rows against a large vocabulary, from the rows and
the vocabulary's weights without keeping the logits, with both gradients.  Rows kept for the way back in 8 bits, restored,
and read by the experts' gradients as they are.  A whole layer of experts for a few tokens: choice, both products, their
weighted sum.

Inputs are made on the GPU from a seed.  `listed` spans one token to training batches, in 32 and 16 bits; `draw` spreads
further cases over the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

#: columns that share a step in rows kept in 8 bits
BLOCK = 32


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def listed():
    return [
        # three positions of an answer are scored: the vocabulary's weights are what is read
        dict(name="xent_score_bf16", op="xent", dtype="bf16", rows=3, vocabulary=131_072, inner=2048, masked=0.0, mode="forward"),
        # a training batch: loss, then both gradients
        dict(name="xent_train_bf16", op="xent", dtype="bf16", rows=4096, vocabulary=65_536, inner=2048, masked=0.0, mode="train"),
        # fine-tuning on answers alone: two fifths of the positions are the question's; an odd vocabulary
        dict(name="xent_masked_f16", op="xent", dtype="f16", rows=2021, vocabulary=100_003, inner=1024, masked=0.4, mode="train"),
        # odd sizes in single precision: rows that no vector load fits
        dict(name="xent_odd_f32", op="xent", dtype="f32", rows=509, vocabulary=10_007, inner=499, masked=0.1, mode="train"),
        # one token of one conversation through gated experts
        dict(name="step_one_bf16", op="step", dtype="bf16", tokens=1, experts=64, top_k=8, inner=2048, hidden=1024, outer=2048,
             act="silu", gated=True, bias=False, residual=True, normalise=True, masked=0.0),
        # sixteen conversations, two wide experts each
        dict(name="step_batch_bf16", op="step", dtype="bf16", tokens=16, experts=32, top_k=2, inner=2048, hidden=4096, outer=2048,
             act="gelu", gated=False, bias=True, residual=True, normalise=True, masked=0.0),
        # odd sizes in single precision, one of the five slots empty
        dict(name="step_odd_f32", op="step", dtype="f32", tokens=5, experts=7, top_k=3, inner=499, hidden=777, outer=501,
             act="relu", gated=False, bias=True, residual=False, normalise=False, masked=0.2),
        # a full server: sixty-four tokens that reach nearly every one of many narrow experts
        dict(name="step_full_f16", op="step", dtype="f16", tokens=64, experts=128, top_k=8, inner=2048, hidden=1024, outer=2048,
             act="silu", gated=True, bias=False, residual=True, normalise=True, masked=0.0),
        # a short sequence's rows kept and restored: latency
        dict(name="kept_short_bf16", op="kept", dtype="bf16", rows=128, inner=2048, mode="restore"),
        # a training batch's wide rows kept and restored
        dict(name="kept_rows_bf16", op="kept", dtype="bf16", rows=16_384, inner=8192, mode="restore"),
        # a layer of experts in training, its input and the rows before the activation kept in 8 bits
        dict(name="kept_experts_bf16", op="kept", dtype="bf16", mode="train", tokens=4096, experts=32, top_k=4, inner=1024, outer=4096,
             act="gelu", bias=True),
        # the way back alone, from rows kept earlier: odd sizes in single precision
        dict(name="kept_odd_f32", op="kept", dtype="f32", mode="backward", tokens=1500, experts=7, top_k=2, inner=499, outer=777,
             act="silu", bias=True),
    ]


def _spread(rng, lo, hi):
    """A whole number from [lo, hi], spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["xent", "xent", "step", "step", "kept"])
    c = dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16", "f16"]))
    single = c["dtype"] == "f32"
    if op == "xent":
        vocabulary, inner = _spread(rng, 1000, 200_000), _spread(rng, 64, 4096)
        if rng.random() < 0.6:
            vocabulary, inner = vocabulary // 64 * 64 + 64, inner // 64 * 64 + 64
        while vocabulary * inner > 1 << 28:
            vocabulary //= 2
        limit = (1 << (36 if single else 39)) // (vocabulary * inner)
        c.update(rows=_spread(rng, 1, max(1, min(8192, limit))), vocabulary=vocabulary, inner=inner, masked=rng.choice([0.0, 0.0, 0.3]),
                 mode=rng.choice(["forward", "train", "train"]))
    elif op == "step":
        experts = _spread(rng, 2, 256)
        inner, hidden, outer = _spread(rng, 64, 4096), _spread(rng, 64, 4096), _spread(rng, 64, 4096)
        if rng.random() < 0.6:
            inner, hidden, outer = (n // 64 * 64 + 32 for n in (inner, hidden, outer))
        while experts * hidden * (2 * inner + outer) > (1 << (28 if single else 29)):
            experts, hidden = max(2, experts // 2), hidden if experts > 2 else hidden // 2
        c.update(tokens=_spread(rng, 1, 64), experts=experts, top_k=rng.randint(1, min(8, experts)), inner=inner, hidden=hidden, outer=outer,
                 act=rng.choice(["none", "relu", "gelu", "silu", "silu"]), gated=rng.random() < 0.5, bias=rng.random() < 0.5,
                 residual=rng.random() < 0.5, normalise=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.2]))
    elif rng.random() < 0.4:
        inner = _spread(rng, 1, 16_384)
        c.update(rows=_spread(rng, 1, min(65_536, (1 << 27) // inner)), inner=inner, mode="restore")
    else:
        # (In 32 bits a kept row of the forward pass may differ by a step where a sum lies next to the border of two: the way
        # back is a case of its own there, from rows kept before.)
        experts, mode = _spread(rng, 2, 64), "backward" if single else rng.choice(["train", "train", "backward"])
        top_k = rng.randint(1, min(4, experts))
        inner, outer = _spread(rng, 64, 2048), _spread(rng, 64, 4096)
        if rng.random() < 0.6:
            inner, outer = inner // 64 * 64 + 32, outer // 64 * 64 + 32
        while experts * inner * outer > 1 << 27:
            experts = max(top_k, experts // 2)
            outer = outer if experts > top_k else outer // 2
        limit = (1 << 36) // (inner * outer * top_k) // (4 if single else 1)
        c.update(tokens=_spread(rng, 1, max(1, min(8192, limit))), experts=experts, top_k=top_k, inner=inner, outer=outer,
                 act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.5, mode=mode)
    return c


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op == "xent":
        rows, v, k = case["rows"], case["vocabulary"], case["inner"]
        held = rows * (1 - case["masked"])
        if case["mode"] == "forward":
            return {"bytes": int((held + v) * k * e + rows * 16), "flops": int(2 * held * v * k)}
        # the gradient's call has no logits: it makes them again from what it reads
        return {"bytes": int((3 * held + rows + 3 * v) * k * e + rows * 28), "flops": int(8 * held * v * k)}
    if op == "step":
        t, n, matrices = case["tokens"], case["experts"], 2 + case["gated"]
        held = t * (1 - case["masked"])
        share = 1 - (1 - case["top_k"] / n) ** held                     # experts that have a token
        weights = n * share * case["hidden"] * (case["inner"] * (1 + case["gated"]) + case["outer"])
        rows = held * case["inner"] + t * case["outer"] * (1 + case["residual"]) + t * n
        sums = case["inner"] * (matrices - 1) + case["outer"]
        return {"bytes": int((weights + rows) * e), "flops": int(2 * held * case["top_k"] * case["hidden"] * sums)}
    if case["mode"] == "restore":
        # rows in, codes and steps out; codes and steps in, rows out
        return {"bytes": int(case["rows"] * case["inner"] * (2 * e + 2 * (1 + 1 / BLOCK))), "flops": int(case["rows"] * case["inner"] * 4)}
    t, k, n = case["tokens"], case["inner"], case["outer"]
    slots, kept = t * case["top_k"], 1 + 1 / BLOCK
    share = 1 - (1 - case["top_k"] / case["experts"]) ** t
    weights, pre = case["experts"] * share * n * k, slots * n * (case["act"] != "none")
    # back: the result's gradient, kept rows and weights in; gradients of rows and weights out
    total = (slots * n + weights + slots * k + case["experts"] * n * k) * e + (t * k + pre) * kept
    if case["mode"] == "train":
        total += (t * k + weights + slots * n) * e + (t * k + pre) * kept
    return {"bytes": int(total), "flops": int(2 * slots * k * n * (3 if case["mode"] == "train" else 2))}


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEVICE) * scale).to(dtype)


def _uniform(g, shape):
    return torch.rand(shape, generator=g, device=DEVICE)


def _grouped(g, tokens, experts, top_k):
    """Bounds of every expert's rows and the token of every row; a few experts are several times as popular as most."""
    liking = torch.randn(experts, generator=g, device=DEVICE) * 0.6
    noise = -torch.log(-torch.log(_uniform(g, (tokens, experts)).clamp(1e-7, 1 - 1e-7)))
    flat = torch.sort(liking + noise, dim=1, descending=True)[1][:, :top_k].reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    counts = torch.zeros(experts, dtype=torch.int64, device=DEVICE).index_add_(0, flat, torch.ones_like(flat))
    bounds = torch.zeros(experts + 1, dtype=torch.int32, device=DEVICE)
    bounds[1:] = torch.cumsum(counts, 0)
    return bounds, (order // top_k).to(torch.int32)


def _inputs(case, seed):
    g, dtype = _generator(seed), DTYPES[case["dtype"]]
    if case["op"] == "xent":
        rows, v, k = case["rows"], case["vocabulary"], case["inner"]
        s = dict(x=_normal(g, (rows, k), dtype), head=torch.empty((v, k), dtype=dtype, device=DEVICE))
        for at in range(0, v, 16_384):
            s["head"][at:at + 16_384] = _normal(g, (min(16_384, v - at), k), dtype, 2.0 * k ** -0.5)
        # frequent tokens come first in a vocabulary
        s["label"] = (_uniform(g, (rows,)).double() ** 3 * v).long().clamp(max=v - 1)
        s["label"][_uniform(g, (rows,)) < case["masked"]] = -100
        # (a program that trains in half precision scales its loss, or small gradients vanish)
        s["weight"] = (0.5 + _uniform(g, (rows,))) * (1024 if dtype is torch.float16 else 1)
        return s
    if case["op"] == "step":
        t, n, k, h, o = case["tokens"], case["experts"], case["inner"], case["hidden"], case["outer"]

        def weights(rows, cols):
            w = torch.empty((n, rows, cols), dtype=dtype, device=DEVICE)
            for e in range(n):
                w[e] = _normal(g, (rows, cols), dtype, cols ** -0.5)
            return w

        bias = lambda rows: _normal(g, (n, rows), dtype, 0.1) if case["bias"] else None
        s = dict(x=_normal(g, (t, k), dtype), logits=_normal(g, (t, n), dtype) + _normal(g, (n,), dtype, 0.5), up=weights(h, k), up_bias=bias(h),
                 down=weights(o, h), down_bias=bias(o), residual=_normal(g, (t, o), dtype) if case["residual"] else None)
        s["gate"], s["gate_bias"] = (weights(h, k), bias(h)) if case["gated"] else (None, None)
        s["keep"] = _uniform(g, (t,)) >= case["masked"] if case["masked"] else None
        return s
    if case["mode"] == "restore":
        # (rows of a network differ in size, and so do stretches of a row)
        rows, k = case["rows"], case["inner"]
        return dict(x=(torch.randn((rows, k), generator=g, device=DEVICE) * torch.exp(torch.randn((rows, 1), generator=g, device=DEVICE))).to(dtype))
    tokens, experts, k, n = case["tokens"], case["experts"], case["inner"], case["outer"]
    bounds, token = _grouped(g, tokens, experts, case["top_k"])
    s = dict(x=_normal(g, (tokens, k), dtype), weight=_normal(g, (experts, n, k), dtype, k ** -0.5), bounds=bounds, token=token,
             bias=_normal(g, (experts, n), dtype, 0.1) if case["bias"] else None, grad_y=_normal(g, (tokens * case["top_k"], n), dtype))
    if case["mode"] == "backward":
        s["x"] = _plain_keep(s["x"])
        s["pre"] = _plain_keep(torch.randn((tokens * case["top_k"], n), generator=g, device=DEVICE)) if case["act"] != "none" else None
    return s


def prepare(case, seed):
    return dict(case=case, **_inputs(case, seed))


# --------------------------------------------------------------------------- #
# the operators in plain form
# --------------------------------------------------------------------------- #
def _plain_xent(s):
    x, head = s["x"].float(), s["head"].float()
    label = s["label"]
    held = (label >= 0) & (label < head.shape[0]) & (s["weight"] != 0)
    at = torch.where(held, label, torch.zeros_like(label))[:, None]
    z = x @ head.t()
    top = z.max(dim=1, keepdim=True)[0]
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(dim=1))
    zero = torch.zeros_like(lse)
    outputs = [torch.where(held, s["weight"] * (lse - torch.gather(z, 1, at)[:, 0]), zero), torch.where(held, lse, zero)]
    if s["case"]["mode"] == "train":
        factor = torch.where(held, s["weight"], zero)[:, None]
        q = torch.exp(z - lse[:, None]).scatter_add_(1, at, torch.full_like(top, -1.0))
        q = q * factor
        outputs += [(q @ head).to(s["x"].dtype), (q.t().contiguous() @ x).to(s["head"].dtype)]
    return outputs


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def _plain_step(s):
    case, k = s["case"], s["case"]["top_k"]
    z = s["logits"].float()
    t, n = z.shape
    keep = s["keep"] if s["keep"] is not None else torch.ones(t, dtype=torch.bool, device=z.device)
    high, best = torch.sort(z, dim=1, descending=True, stable=True)
    p = torch.exp(high[:, :k] - high[:, :1])
    whole = p.sum(dim=1, keepdim=True) if case["normalise"] else torch.exp(z - high[:, :1]).sum(dim=1, keepdim=True)
    share = torch.where(keep[:, None], p / whole, torch.zeros_like(p))          # [t, k], of the experts `best`
    x, choice = s["x"].float(), best[:, :k]
    bias = lambda b: b.float()[choice] if b is not None else 0.0
    if t * k <= n:
        # few rows: the weights of every (token, choice)
        into = lambda w: torch.bmm(w[choice.reshape(-1)].float(), x[:, None].expand(t, k, -1).reshape(t * k, -1, 1)).reshape(t, k, -1)
        out_of = lambda h: torch.bmm(s["down"][choice.reshape(-1)].float(), h.reshape(t * k, -1, 1)).reshape(t, k, -1)
    else:
        # every expert with every token, of which the chosen ones are taken
        into = lambda w: torch.gather((x @ w.float().reshape(-1, x.shape[1]).t()).reshape(t, n, -1), 1, choice[:, :, None].expand(-1, -1, w.shape[1]))

        def out_of(h):
            rows = torch.zeros((t, n, h.shape[2]), device=h.device).scatter_(1, choice[:, :, None].expand(-1, -1, h.shape[2]), h)
            y = torch.bmm(rows.transpose(0, 1).contiguous(), s["down"].float().transpose(1, 2).contiguous()).transpose(0, 1)
            return torch.gather(y, 1, choice[:, :, None].expand(-1, -1, y.shape[2]))

    h = into(s["up"]) + bias(s["up_bias"])
    if s["gate"] is not None:
        h = _act(into(s["gate"]) + bias(s["gate_bias"]), case["act"]) * h
    else:
        h = _act(h, case["act"])
    out = ((out_of(h) + bias(s["down_bias"])) * share[:, :, None]).sum(dim=1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return [out.to(s["x"].dtype)]


def _power_of_two(exponent):
    """(From the exponent's bits: a power that is off by its last one would move values halfway between two codes.)"""
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def _plain_keep(x):
    """Codes and exponents of rows kept in 8 bits: a block's step is a power of two, with which its largest value has 64 to
    127 of them.  (The exponent is stored with 127 added.)"""
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    v = torch.zeros((rows, blocks * BLOCK), device=x.device)
    v[:, :cols] = x.float()
    v = v.reshape(rows, blocks, BLOCK)
    exponent = torch.frexp(v.abs().max(dim=2)[0])[1] - 7
    exponent = torch.where((v == 0).all(dim=2), torch.full_like(exponent, -127), exponent.clamp(min=-127))
    codes = torch.round(v.double() / _power_of_two(exponent)[:, :, None]).clamp(-127, 127).to(torch.int8)
    return codes.reshape(rows, -1)[:, :cols].contiguous(), (exponent + 127).to(torch.uint8)


def _plain_restore(kept):
    codes, exponent = kept
    step = _power_of_two(exponent.long() - 127).repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]
    return (codes.double() * step).float()


def _plain_kept(s):
    case = s["case"]
    if case["mode"] == "restore":
        return [_plain_restore(_plain_keep(s["x"])).to(s["x"].dtype)]
    # the groups of rows side by side, padded to the longest: one batched product for all experts
    bounds, token, dtype = s["bounds"].long(), s["token"].long(), s["grad_y"].dtype
    slots = torch.arange(token.numel(), device=token.device)
    expert = torch.searchsorted(bounds[1:].contiguous(), slots, right=True)
    place = slots - bounds[expert]
    longest = int((bounds[1:] - bounds[:-1]).max())
    w = s["weight"].float()
    side_by_side = lambda v: torch.zeros((w.shape[0], longest, v.shape[1]), device=v.device).index_put_((expert, place), v)
    outputs = []
    if case["mode"] == "train":
        z = torch.bmm(side_by_side(s["x"].float()[token]), w.transpose(1, 2))[expert, place]
        if s["bias"] is not None:
            z = z + s["bias"].float()[expert]
        outputs.append(_act(z, case["act"]).to(dtype))
        x, pre = _plain_restore(_plain_keep(s["x"])), _plain_restore(_plain_keep(z)) if case["act"] != "none" else None
    else:
        x, pre = _plain_restore(s["x"]), _plain_restore(s["pre"]) if s["pre"] is not None else None
    grad_z = s["grad_y"].float()
    if pre is not None:
        grad_z = grad_z * _act_slope(pre, case["act"])
    grad_z = side_by_side(grad_z)
    outputs.append(torch.bmm(grad_z, w)[expert, place].to(dtype))
    outputs.append(torch.bmm(grad_z.transpose(1, 2).contiguous(), side_by_side(x[token])).to(dtype))
    if s["bias"] is not None:
        outputs.append(grad_z.sum(dim=1).to(dtype))
    return outputs


# --------------------------------------------------------------------------- #
# the library's operators
# --------------------------------------------------------------------------- #
def _own_xent(s):
    from paper_2604_17198_amd import binding as nb
    loss, lse = nb.nacho_xent(s["x"], s["head"], s["label"], weight=s["weight"])
    if s["case"]["mode"] == "forward":
        return [loss, lse]
    return [loss, lse, *nb.nacho_xent_grad(s["x"], s["head"], s["label"], lse, weight=s["weight"])]


def _own_step(s):
    from paper_2604_17198_amd import binding as nb
    case = s["case"]
    return [nb.nacho_experts_step(s["x"], s["logits"], case["top_k"], s["up"], s["down"], gate=s["gate"], up_bias=s["up_bias"],
                                  gate_bias=s["gate_bias"], down_bias=s["down_bias"], act=case["act"], normalise=case["normalise"],
                                  keep=s["keep"], residual=s["residual"])]


def _own_kept(s):
    from paper_2604_17198_amd import binding as nb
    case = s["case"]
    if case["mode"] == "restore":
        return [nb.nacho_restore8(nb.nacho_keep8(s["x"]), s["x"].dtype)]
    more = dict(token=s["token"], act=case["act"])
    outputs = []
    if case["mode"] == "train":
        pre = nb.Kept8.empty(*s["grad_y"].shape, s["x"].device) if case["act"] != "none" else None
        outputs.append(nb.nacho_experts(s["x"], s["weight"], s["bounds"], bias=s["bias"], pre=pre, **more))
        x = nb.nacho_keep8(s["x"])
    else:
        x, pre = nb.Kept8(*s["x"]), nb.Kept8(*s["pre"]) if s["pre"] is not None else None
    grad_bias = torch.empty_like(s["bias"]) if s["bias"] is not None else None
    outputs += nb.nacho_experts_grad(s["grad_y"], x, s["weight"], s["bounds"], pre=pre, grad_bias=grad_bias, **more)
    return outputs + ([grad_bias] if grad_bias is not None else [])


def run(state):
    op = state["case"]["op"]
    if own:
        return {"xent": _own_xent, "step": _own_step, "kept": _own_kept}[op](state)
    return {"xent": _plain_xent, "step": _plain_step, "kept": _plain_kept}[op](state)


# --------------------------------------------------------------------------- #
# the definitions, in 64 bits
# --------------------------------------------------------------------------- #
def _exact_xent(case, s):
    rows, v, train = case["rows"], case["vocabulary"], case["mode"] == "train"
    head = s["head"].double()
    loss = torch.zeros(rows, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros_like(loss)
    grad_x = torch.zeros((rows, case["inner"]), dtype=torch.float64, device=DEVICE)
    grad_head = torch.zeros_like(head) if train else None
    counted = [i for i, l in enumerate(s["label"].tolist()) if 0 <= l < v]
    for at in range(0, len(counted), 512):
        part = torch.tensor(counted[at:at + 512], device=DEVICE)
        x, w, label = s["x"][part].double(), s["weight"][part].double(), s["label"][part]
        z = torch.matmul(x, head.T)
        log_q = torch.log_softmax(z, dim=1)
        loss[part] = -w * log_q[torch.arange(len(part), device=DEVICE), label]
        lse[part] = torch.logsumexp(z, dim=1)
        if train:
            d = torch.exp(log_q)
            d[torch.arange(len(part), device=DEVICE), label] -= 1.0
            d *= w[:, None]
            grad_x[part] = torch.matmul(d, head)
            grad_head += torch.matmul(d.T, x)
    return [loss, lse] + ([grad_x, grad_head] if train else [])


def _exact_act(z, act):
    if act == "gelu":
        return torch.nn.functional.gelu(z)
    if act == "silu":
        return torch.nn.functional.silu(z)
    return torch.relu(z) if act == "relu" else z


def _exact_slope(z, act):
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    return (z > 0).double() if act == "relu" else torch.ones_like(z)


def _exact_step(case, s):
    z = s["logits"].double()
    # an expert's rank in a row: how many are higher, or as high with a lower index
    rank = torch.argsort(torch.argsort(z, dim=1, descending=True, stable=True), dim=1)
    member = rank < case["top_k"]
    if s["keep"] is not None:
        member &= s["keep"][:, None]
    gate = torch.where(member, torch.softmax(z, dim=1), torch.zeros_like(z))
    if case["normalise"]:
        gate = gate / gate.sum(dim=1, keepdim=True).clamp(min=1e-300)
    out = s["residual"].double() if s["residual"] is not None else torch.zeros((case["tokens"], case["outer"]), dtype=torch.float64, device=DEVICE)
    out = out.clone()
    for e in range(case["experts"]):
        tokens = member[:, e].nonzero()[:, 0]
        if tokens.numel() == 0:
            continue

        def layer(rows, w, b):
            y = torch.matmul(rows, s[w][e].double().T)
            return y + s[b][e].double() if s[b] is not None else y

        rows = s["x"][tokens].double()
        h = layer(rows, "up", "up_bias")
        h = _exact_act(layer(rows, "gate", "gate_bias"), case["act"]) * h if case["gated"] else _exact_act(h, case["act"])
        out[tokens] += layer(h, "down", "down_bias") * gate[tokens, e][:, None]
    return [out]


def _exact_kept_rows(x):
    """What rows kept in 8 bits stand for: multiples of a power of two, with the exponent of the block's largest value."""
    x = x.double()
    out = torch.empty_like(x)
    powers = torch.tensor([math.ldexp(1.0, i) for i in range(-127, 129)], dtype=torch.float64, device=DEVICE)
    for at in range(0, x.shape[1], BLOCK):
        part = x[:, at:at + BLOCK]
        largest = part.abs().amax(dim=1, keepdim=True)
        exponent = ((largest.view(torch.int64) >> 52) - 1023 - 6).clamp(min=-127)
        step = powers[exponent + 127]
        out[:, at:at + BLOCK] = torch.minimum(torch.maximum(torch.round(part / step), torch.tensor(-127.0, device=DEVICE)), torch.tensor(127.0, device=DEVICE)) * step
    return out


def _exact_codes(kept):
    codes, exponent = kept
    at = torch.arange(codes.shape[1], device=DEVICE) // BLOCK
    powers = torch.tensor([math.ldexp(1.0, i) for i in range(-127, 129)], dtype=torch.float64, device=DEVICE)
    return codes.double() * powers[exponent.long()][:, at]


def _exact_kept(case, s):
    if case["mode"] == "restore":
        return [_exact_kept_rows(s["x"])]
    train, act, token, bounds = case["mode"] == "train", case["act"], s["token"].long(), s["bounds"].tolist()
    x = _exact_kept_rows(s["x"]) if train else _exact_codes(s["x"])
    parts = []
    for e in range(case["experts"]):
        at = slice(bounds[e], bounds[e + 1])
        w, part, pre = s["weight"][e].double(), [], None
        if train:
            z = torch.matmul(s["x"][token[at]].double(), w.T)
            if s["bias"] is not None:
                z = z + s["bias"][e].double()
            part.append(_exact_act(z, act))
            pre = _exact_kept_rows(z) if act != "none" else None
        elif act != "none":
            pre = _exact_codes((s["pre"][0][at], s["pre"][1][at]))
        gz = s["grad_y"][at].double()
        if pre is not None:
            gz = gz * _exact_slope(pre, act)
        part += [torch.matmul(gz, w), torch.matmul(gz.T, x[token[at]])[None], gz.sum(dim=0)[None]]
        parts.append(part)
    outputs = [torch.cat(column) for column in zip(*parts)]
    return outputs if s["bias"] is not None else outputs[:-1]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"xent": _exact_xent, "step": _exact_step, "kept": _exact_kept}[case["op"]](case, s)
