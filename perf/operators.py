"""The operators of a mixture-of-experts layer and of its distillation, as timed cases.

Four operators over sparse matrices that training makes by itself, each forward and backward: the distillation loss
against a teacher's top logits (a CSR matrix of tokens x vocabulary), the routing of tokens to experts (a CSR matrix of
tokens x experts, its transpose, counts and the balance loss), the experts' products over the ragged groups of rows that
the routing leaves, and the weighted sum of the experts' rows for every token.

Inputs are made on the GPU from a seed.  Logits are normal; popular experts draw several times the tokens of the
others; a teacher's top logits lie in a random subset of the vocabulary, sorted.  `listed` spans single decoding steps to
training batches, in 32 and 16 bits; `draw` spreads further cases over the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def listed():
    return [
        # a handful of positions against a large vocabulary: an online check of the student, loss and gradient
        dict(name="distill_few_rows_f32", op="distill", dtype="f32", rows=4, cols=131_072, least=64, most=64,
             masked=0.0, temperature=1.0, mode="both"),
        # a training batch: every position has the teacher's 64 top logits
        dict(name="distill_train_bf16", op="distill", dtype="bf16", rows=4096, cols=65_536, least=64, most=64,
             masked=0.0, temperature=2.0, mode="both"),
        # an odd vocabulary, rows cut at a probability (none to 512 stored), a fifth padding; the loss first, its gradient later
        dict(name="distill_ragged_f16", op="distill", dtype="f16", rows=1021, cols=100_003, least=0, most=512,
             masked=0.2, temperature=1.5, mode="split"),
        # a decoding step of sixteen sequences
        dict(name="route_step_bf16", op="route", dtype="bf16", tokens=16, experts=64, top_k=8, masked=0.0, closed=0.0,
             normalise=True, mode="forward"),
        # a training batch: routing, balance loss and the gradient of both
        dict(name="route_train_f32", op="route", dtype="f32", tokens=65_536, experts=128, top_k=8, masked=0.0,
             closed=0.0, normalise=True, mode="train"),
        # padding among the tokens and experts closed to some of them, gates not normalised
        dict(name="route_masked_bf16", op="route", dtype="bf16", tokens=10_007, experts=60, top_k=3, masked=0.1,
             closed=0.1, normalise=False, mode="train"),
        # a decoding step: eight tokens, two experts each, the weights are what is read
        dict(name="experts_step_bf16", op="experts", dtype="bf16", tokens=8, experts=32, top_k=2, inner=2048,
             outer=4096, act="gelu", bias=True, mode="forward"),
        # a prefill batch through wide experts
        dict(name="experts_forward_bf16", op="experts", dtype="bf16", tokens=8192, experts=16, top_k=2, inner=2048,
             outer=8192, act="silu", bias=False, mode="forward"),
        # a training batch over many narrow experts, all gradients
        dict(name="experts_train_bf16", op="experts", dtype="bf16", tokens=4096, experts=32, top_k=4, inner=1024,
             outer=4096, act="gelu", bias=True, mode="train"),
        # odd sizes in single precision: rows that no vector load fits
        dict(name="experts_odd_f32", op="experts", dtype="f32", tokens=1500, experts=7, top_k=2, inner=499, outer=777,
             act="relu", bias=True, mode="train"),
        # a decoding step: the experts' rows into the residual stream
        dict(name="combine_step_bf16", op="combine", dtype="bf16", tokens=8, top_k=2, outer=4096, residual=True,
             mode="forward"),
        # a training batch, with the gradients of rows and gates
        dict(name="combine_train_bf16", op="combine", dtype="bf16", tokens=16_384, top_k=4, outer=4096, residual=True,
             mode="train"),
    ]


def _spread(rng, lo, hi):
    """A whole number from [lo, hi], spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["distill", "route", "experts", "experts", "combine"])
    c = dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16", "f16"]))
    if op == "distill":
        cols = _spread(rng, 1000, 200_000)
        most = _spread(rng, 1, 512)
        c.update(rows=_spread(rng, 1, min(8192, (1 << 27) // cols)), cols=cols, least=rng.choice([0, 1, most]), most=most,
                 masked=rng.choice([0.0, 0.2]), temperature=rng.choice([1.0, 1.5, 2.0]),
                 mode=rng.choice(["both", "both", "split", "forward"]))
    elif op == "route":
        experts = _spread(rng, 4, 512)
        c.update(tokens=_spread(rng, 1, min(65_536, (1 << 23) // experts)), experts=experts,
                 top_k=rng.randint(1, min(8, experts)), masked=rng.choice([0.0, 0.1]), closed=rng.choice([0.0, 0.1]),
                 normalise=rng.random() < 0.5, mode=rng.choice(["forward", "train", "train"]))
    elif op == "experts":
        experts, mode = _spread(rng, 2, 64), rng.choice(["forward", "train"])
        top_k = rng.randint(1, min(4, experts))
        inner, outer = _spread(rng, 64, 4096), _spread(rng, 64, 8192)
        if rng.random() < 0.6:
            inner, outer = inner // 64 * 64 + 32, outer // 64 * 64 + 32
        while experts * inner * outer > 1 << 28:
            experts = max(top_k, experts // 2)
            outer = outer if experts > top_k else outer // 2
        limit = (1 << 38) // (inner * outer * top_k) // (3 if mode == "train" else 1)
        if c["dtype"] == "f32":
            limit //= 8
        c.update(tokens=_spread(rng, 1, max(1, min(8192, limit))), experts=experts, top_k=top_k, inner=inner, outer=outer,
                 act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.5, mode=mode)
    else:
        top_k, outer = rng.randint(1, 8), _spread(rng, 64, 8192)
        c.update(tokens=_spread(rng, 1, min(32_768, (1 << 27) // (outer * top_k))), top_k=top_k, outer=outer,
                 residual=rng.random() < 0.5, mode=rng.choice(["forward", "train"]))
    return c


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    op, train = case["op"], case["mode"] == "train"
    if op == "distill":
        # rows of weight zero are not read; the loss and its gradient read the logits once between them, or once each
        rows, held = case["rows"], case["rows"] * (1 - case["masked"])
        stored = (case["least"] + case["most"]) / 2 * rows
        reads, writes = {"both": (1, 1), "split": (2, 1), "forward": (1, 0)}[case["mode"]]
        return {"bytes": int(case["cols"] * e * (held * reads + rows * writes) + stored * 8 * reads + rows * 20),
                "flops": int(held * case["cols"] * 4 * max(1, writes + 1))}
    if op == "route":
        t, experts = case["tokens"], case["experts"]
        entries = t * case["top_k"]
        # forward: logits in; experts, gates, places and tokens out.  Backward: logits, entries and gates' gradients in
        total = t * experts * e + entries * 16 + t * 8
        if train:
            total += 2 * t * experts * e + entries * 12 + t * 8
        return {"bytes": int(total), "flops": int(t * experts * (4 + case["top_k"]) * (2 if train else 1))}
    if op == "experts":
        t, k, n = case["tokens"], case["inner"], case["outer"]
        slots = t * case["top_k"]
        share = 1 - (1 - case["top_k"] / case["experts"]) ** t            # experts that have a row
        weights = case["experts"] * share * n * k
        total = t * k + weights + slots * n
        if train:
            # the rows before the activation out and in; gradients of rows and weights out, of the result in
            total += 2 * slots * n * (case["act"] != "none") + slots * n + weights + t * k + slots * k + case["experts"] * n * k
        return {"bytes": int(total * e), "flops": int(2 * slots * k * n * (3 if train else 1))}
    t, n = case["tokens"], case["outer"]
    slots = t * case["top_k"]
    total = (slots + t * (1 + case["residual"])) * n * e + slots * 8
    if train:
        total += (t + 2 * slots) * n * e + slots * 12
    return {"bytes": int(total), "flops": int(slots * n * (5 if train else 2))}


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


def _chosen(g, tokens, experts, top_k):
    """[tokens, top_k] distinct experts a token, ascending; a few experts are several times as popular as most."""
    liking = torch.randn(experts, generator=g, device=DEVICE) * 0.6
    noise = -torch.log(-torch.log(_uniform(g, (tokens, experts)).clamp(1e-7, 1 - 1e-7)))
    return torch.sort(torch.sort(liking + noise, dim=1, descending=True)[1][:, :top_k], dim=1)[0]


def _grouped(chosen, experts):
    """Bounds of every expert's rows, the token of every row, and the row of every (token, choice)."""
    tokens, top_k = chosen.shape
    flat = chosen.reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    counts = torch.zeros(experts, dtype=torch.int64, device=DEVICE).index_add_(0, flat, torch.ones_like(flat))
    bounds = torch.zeros(experts + 1, dtype=torch.int32, device=DEVICE)
    bounds[1:] = torch.cumsum(counts, 0)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(order.numel(), device=DEVICE)
    return bounds, (order // top_k).to(torch.int32), slot.to(torch.int32)


def _inputs(case, seed):
    g, dtype = _generator(seed), DTYPES[case["dtype"]]
    if case["op"] == "distill":
        rows, cols = case["rows"], case["cols"]
        s = dict(logits=torch.empty((rows, cols), dtype=dtype, device=DEVICE))
        for at in range(0, rows, 256):                      # (a stretch at a time: noise in 32 bits is twice the logits)
            s["logits"][at:at + 256] = _normal(g, (min(256, rows - at), cols), dtype, 2.0)
        held = torch.randint(case["least"], case["most"] + 1, (rows,), generator=g, device=DEVICE)
        held = torch.clamp(held, max=cols)
        pos = torch.zeros(rows + 1, dtype=torch.int32, device=DEVICE)
        pos[1:] = torch.cumsum(held, 0)
        # stored columns: one in each of `held` equal stretches of the vocabulary, sorted by construction
        row = torch.repeat_interleave(torch.arange(rows, device=DEVICE), held)
        i = torch.arange(row.numel(), device=DEVICE) - pos[row].long()
        lo, hi = i * cols // held[row], (i + 1) * cols // held[row]
        crd = lo + (_uniform(g, (row.numel(),)) * (hi - lo)).long().clamp(max=cols)
        s["pos"], s["crd"] = pos, torch.minimum(crd, hi - 1).to(torch.int32)
        s["val"] = s["logits"][row, s["crd"].long()].float() + _normal(g, (row.numel(),), torch.float32) + 6.0
        # (a program that trains in half precision scales its loss, or small gradients vanish)
        weight = (0.5 + _uniform(g, (rows,))) * (1024 if dtype is torch.float16 else 1)
        s["weight"] = torch.where(_uniform(g, (rows,)) < case["masked"], torch.zeros_like(weight), weight)
        return s
    if case["op"] == "route":
        tokens, experts = case["tokens"], case["experts"]
        logits = torch.randn((tokens, experts), generator=g, device=DEVICE) + torch.randn(experts, generator=g, device=DEVICE) * 0.5
        closed = _uniform(g, (tokens, experts)) < case["closed"]
        closed[:, 0] = False                                # (one expert takes every token)
        s = dict(logits=torch.where(closed, torch.full_like(logits, -math.inf), logits).to(dtype))
        s["keep"] = _uniform(g, (tokens,)) >= case["masked"] if case["masked"] else None
        s["grad_gate"] = _normal(g, (tokens * case["top_k"],), torch.float32)
        return s
    if case["op"] == "experts":
        tokens, experts, k, n = case["tokens"], case["experts"], case["inner"], case["outer"]
        bounds, token, _ = _grouped(_chosen(g, tokens, experts, case["top_k"]), experts)
        return dict(x=_normal(g, (tokens, k), dtype), weight=_normal(g, (experts, n, k), dtype, k ** -0.5),
                    bias=_normal(g, (experts, n), dtype, 0.1) if case["bias"] else None, bounds=bounds, token=token,
                    grad_y=_normal(g, (tokens * case["top_k"], n), dtype) if case["mode"] == "train" else None)
    tokens, top_k, n = case["tokens"], case["top_k"], case["outer"]
    _, _, slot = _grouped(_chosen(g, tokens, 2 * top_k + 8, top_k), 2 * top_k + 8)
    return dict(y=_normal(g, (tokens * top_k, n), dtype), pos=torch.arange(tokens + 1, dtype=torch.int32, device=DEVICE) * top_k,
                slot=slot, gate=_uniform(g, (tokens * top_k,)), residual=_normal(g, (tokens, n), dtype) if case["residual"] else None,
                grad_out=_normal(g, (tokens, n), dtype) if case["mode"] == "train" else None)


def prepare(case, seed):
    return dict(case=case, **_inputs(case, seed))


# --------------------------------------------------------------------------- #
# the operators in plain form
# --------------------------------------------------------------------------- #
def _softmax_stats(z):
    """max and log of the sum of exponentials of every row."""
    top = z.max(dim=1, keepdim=True)[0]
    return top[:, 0] + torch.log(torch.exp(z - top).sum(dim=1))


def _plain_distill(s):
    case, tau = s["case"], s["case"]["temperature"]
    z = s["logits"].float() / tau
    rows = z.shape[0]
    held = (s["pos"][1:] - s["pos"][:-1]).long()
    row = torch.repeat_interleave(torch.arange(rows, device=z.device), held, output_size=s["crd"].numel())
    col = s["crd"].long()
    active = (held > 0) & (s["weight"] != 0)
    lse = _softmax_stats(z)
    u = s["val"] / tau
    top = torch.full((rows,), -math.inf, device=z.device).index_reduce_(0, row, u, "amax")
    total = torch.zeros(rows, device=z.device).index_add_(0, row, torch.exp(u - top[row]))
    log_p = u - top[row] - torch.log(total)[row]
    log_q = z[row, col] - lse[row]
    p = torch.exp(log_p)
    loss = torch.zeros(rows, device=z.device).index_add_(0, row, p * (log_p - log_q)) * s["weight"] * tau * tau
    zero = torch.zeros_like(loss)
    outputs = [torch.where(active, loss, zero), torch.where(active, lse, zero)]
    if case["mode"] != "forward":
        scale = torch.where(active, s["weight"] * tau, zero)
        q = torch.exp(z - lse[:, None])
        q[row, col] -= p
        outputs.append((q * scale[:, None]).to(s["logits"].dtype))
    return outputs


def _plain_route(s):
    case, k = s["case"], s["case"]["top_k"]
    z = s["logits"].float()
    tokens, experts = z.shape
    keep = s["keep"] if s["keep"] is not None else torch.ones(tokens, dtype=torch.bool, device=z.device)
    lse = torch.where(keep, _softmax_stats(z), torch.zeros(tokens, device=z.device))
    p = torch.where(keep[:, None], torch.exp(z - lse[:, None]), torch.zeros_like(z))
    high, best = torch.sort(z, dim=1, descending=True, stable=True)
    taken = (high[:, :k] > -math.inf) & keep[:, None]
    choice = torch.sort(torch.where(taken, best[:, :k], torch.full_like(best[:, :k], experts)), dim=1)[0]
    taken = choice < experts
    gate = torch.where(taken, torch.gather(p, 1, choice.clamp(max=experts - 1)), torch.zeros_like(high[:, :k]))
    whole = gate.sum(dim=1, keepdim=True)
    if case["normalise"]:
        gate = torch.where(taken, gate / whole, gate)
    pos = torch.zeros(tokens + 1, dtype=torch.int32, device=z.device)
    pos[1:] = torch.cumsum(taken.sum(dim=1), 0)
    # the entries in a row, absent ones moved behind them; then by expert, tokens ascending
    flat = torch.sort((~taken).reshape(-1).to(torch.int8), stable=True)[1]
    expert = torch.where(taken, choice, torch.full_like(choice, experts)).reshape(-1)[flat]
    order = torch.sort(expert, stable=True)[1]
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=z.device).index_add_(0, expert, torch.ones_like(expert))[:experts]
    expert_pos = torch.zeros(experts + 1, dtype=torch.int32, device=z.device)
    expert_pos[1:] = torch.cumsum(counts, 0)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(order.numel(), device=z.device)
    absent = expert == experts
    none = torch.full_like(expert, -1)
    token = torch.where(absent[order], none, (flat // k)[order])
    entries, routed = counts.sum(), taken.any(dim=1).sum()
    share = counts.float() / entries.clamp(min=1)
    balance = experts * (share * p.sum(dim=0) / routed.clamp(min=1)).sum()
    outputs = [pos, torch.where(absent, none, expert).to(torch.int32), gate.reshape(-1)[flat],
               torch.where(absent, none, slot).to(torch.int32), expert_pos, token.to(torch.int32), counts.to(torch.int32),
               lse, balance.reshape(1)]
    if case["mode"] == "train":
        dg = torch.zeros(tokens * k, device=z.device)
        dg[flat] = torch.where(absent, torch.zeros_like(s["grad_gate"]), s["grad_gate"])
        dg = dg.reshape(tokens, k)
        inner = (gate * dg).sum(dim=1, keepdim=True)
        index = choice.clamp(max=experts - 1)
        chosen = torch.where(taken, gate * (dg - inner) if case["normalise"] else gate * dg, torch.zeros_like(gate))
        grad = torch.zeros_like(z).scatter_add_(1, index, chosen)
        if not case["normalise"]:
            grad -= p * inner
        c = BALANCE * experts * share / routed.clamp(min=1)
        grad += p * (c - (p * c).sum(dim=1, keepdim=True))
        outputs.append(grad.to(s["logits"].dtype))
    return outputs


#: weight of the balance loss in the training objective
BALANCE = 0.01


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


def _plain_experts(s):
    # the groups of rows side by side, padded to the longest: one batched product for all experts
    case, x, bounds = s["case"], s["x"], s["bounds"].long()
    slots = torch.arange(s["token"].numel(), device=x.device)
    expert = torch.searchsorted(bounds[1:].contiguous(), slots, right=True)
    place = slots - bounds[expert]
    longest = int((bounds[1:] - bounds[:-1]).max())
    w = s["weight"].float()
    rows = torch.zeros((w.shape[0], longest, x.shape[1]), device=x.device)
    rows[expert, place] = x[s["token"].long()].float()
    z = torch.bmm(rows, w.transpose(1, 2))[expert, place]
    if s["bias"] is not None:
        z = z + s["bias"].float()[expert]
    outputs = [_act(z, case["act"]).to(x.dtype)]
    if case["mode"] == "train":
        grad_z = torch.zeros((w.shape[0], longest, w.shape[1]), device=x.device)
        grad_z[expert, place] = s["grad_y"].float() * _act_slope(z, case["act"])
        outputs.append(torch.bmm(grad_z, w)[expert, place].to(x.dtype))
        outputs.append(torch.bmm(grad_z.transpose(1, 2).contiguous(), rows).to(x.dtype))
        if s["bias"] is not None:
            outputs.append(grad_z.sum(dim=1).to(x.dtype))
    return outputs


def _plain_combine(s):
    case, y = s["case"], s["y"]
    tokens, top_k = s["pos"].numel() - 1, case["top_k"]
    slot = s["slot"].long()
    rows = y[slot].float().reshape(tokens, top_k, -1)
    gate = s["gate"].reshape(tokens, top_k, 1)
    out = (rows * gate).sum(dim=1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    outputs = [out.to(y.dtype)]
    if case["mode"] == "train":
        go = s["grad_out"].float()[:, None, :]
        grad_y = torch.empty_like(y)
        grad_y[slot] = (go * gate).to(y.dtype).reshape(tokens * top_k, -1)
        outputs += [grad_y, (go * rows).sum(dim=2).reshape(-1)]
    return outputs


# --------------------------------------------------------------------------- #
# the library's operators
# --------------------------------------------------------------------------- #
def _own_distill(s):
    from paper_2604_17198_amd import binding as nb
    case, z = s["case"], s["logits"]
    teacher = nb.csr(s["pos"], s["crd"], z.shape[0], z.shape[1], s["val"])
    more = dict(temperature=case["temperature"], weight=s["weight"])
    if case["mode"] == "both":
        grad = torch.empty_like(z)
        loss, lse = nb.nacho_distill(teacher, z, grad=grad, **more)
        return [loss, lse, grad]
    loss, lse = nb.nacho_distill(teacher, z, **more)
    if case["mode"] == "forward":
        return [loss, lse]
    return [loss, lse, nb.nacho_distill_grad(teacher, z, lse, **more)]


def _own_route(s):
    from paper_2604_17198_amd import binding as nb
    case, z = s["case"], s["logits"]
    r = nb.nacho_route(z, case["top_k"], normalise=case["normalise"], keep=s["keep"])
    outputs = [r.pos, r.expert, r.gate, r.slot, r.expert_pos, r.token, r.counts, r.lse, r.balance]
    if case["mode"] == "train":
        outputs.append(nb.nacho_route_grad(z, r, s["grad_gate"], balance=BALANCE, keep=s["keep"]))
    return outputs


def _own_experts(s):
    from paper_2604_17198_amd import binding as nb
    case = s["case"]
    more = dict(token=s["token"], act=case["act"])
    if case["mode"] == "forward":
        return [nb.nacho_experts(s["x"], s["weight"], s["bounds"], bias=s["bias"], **more)]
    # the rows before the activation are kept for the way back
    pre = torch.empty_like(s["grad_y"]) if case["act"] != "none" else None
    y = nb.nacho_experts(s["x"], s["weight"], s["bounds"], bias=s["bias"], pre=pre, **more)
    grad_bias = torch.empty_like(s["bias"]) if s["bias"] is not None else None
    grad_x, grad_weight = nb.nacho_experts_grad(s["grad_y"], s["x"], s["weight"], s["bounds"], pre=pre, grad_bias=grad_bias, **more)
    return [y, grad_x, grad_weight] + ([grad_bias] if grad_bias is not None else [])


def _own_combine(s):
    from paper_2604_17198_amd import binding as nb
    outputs = [nb.nacho_combine(s["pos"], s["slot"], s["y"], gate=s["gate"], residual=s["residual"])]
    if s["case"]["mode"] == "train":
        outputs += nb.nacho_combine_grad(s["pos"], s["slot"], s["y"], s["grad_out"], gate=s["gate"])
    return outputs


def run(state):
    op = state["case"]["op"]
    if own:
        return {"distill": _own_distill, "route": _own_route, "experts": _own_experts, "combine": _own_combine}[op](state)
    return {"distill": _plain_distill, "route": _plain_route, "experts": _plain_experts, "combine": _plain_combine}[op](state)


# --------------------------------------------------------------------------- #
# the definitions, in 64 bits
# --------------------------------------------------------------------------- #
def _exact_distill(case, s):
    tau, pos = case["temperature"], s["pos"].tolist()
    loss, lse = torch.zeros(case["rows"], dtype=torch.float64), torch.zeros(case["rows"], dtype=torch.float64)
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device=DEVICE) if case["mode"] != "forward" else None
    weight = s["weight"].double().tolist()
    for at in range(0, case["rows"], 256):
        rows = [i for i in range(at, min(at + 256, case["rows"])) if weight[i] != 0 and pos[i + 1] > pos[i]]
        if not rows:
            continue
        z = s["logits"][rows].double() / tau
        log_q = torch.log_softmax(z, dim=1)
        norm = torch.logsumexp(z, dim=1)
        teacher = torch.full_like(z, -math.inf)
        which = torch.cat([torch.full((pos[i + 1] - pos[i],), n, device=DEVICE) for n, i in enumerate(rows)])
        held = torch.cat([torch.arange(pos[i], pos[i + 1], device=DEVICE) for i in rows])
        teacher[which, s["crd"][held].long()] = s["val"][held].double() / tau
        log_p = torch.log_softmax(teacher, dim=1)
        p = torch.exp(log_p)
        w = s["weight"][rows].double()
        loss[rows] = (torch.where(p > 0, p * (log_p - log_q), torch.zeros_like(p)).sum(dim=1) * w * tau * tau).cpu()
        lse[rows] = norm.cpu()
        if grad is not None:
            grad[rows] = (torch.exp(log_q) - p) * (w * tau)[:, None]
    return [loss, lse] + ([grad] if grad is not None else [])


def _exact_route(case, s):
    z, k, experts = s["logits"].double().cpu(), case["top_k"], case["experts"]
    tokens = z.shape[0]
    keep = s["keep"].cpu() if s["keep"] is not None else torch.ones(tokens, dtype=torch.bool)
    p = torch.where(keep[:, None], torch.softmax(z, dim=1), torch.zeros_like(z))
    lse = torch.where(keep, torch.logsumexp(z, dim=1), torch.zeros(tokens, dtype=torch.float64))
    # an expert's rank in a row: how many are higher, or as high with a lower index
    rank = torch.argsort(torch.argsort(z, dim=1, descending=True, stable=True), dim=1)
    member = (rank < k) & (z > -math.inf) & keep[:, None]
    gate = torch.where(member, p, torch.zeros_like(p))
    if case["normalise"]:
        gate = gate / gate.sum(dim=1, keepdim=True).clamp(min=1e-300)
    where = member.nonzero()
    entries, room = where.shape[0], tokens * k

    def padded(v, fill):
        full = torch.full((room,), fill, dtype=v.dtype)
        full[:entries] = v
        return full

    bounds = lambda m: torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(m, 0)]).to(torch.int32)
    by_expert = member.t().nonzero()
    number = torch.zeros((tokens, experts), dtype=torch.int64)
    number[by_expert[:, 1], by_expert[:, 0]] = torch.arange(entries)
    counts, routed = member.sum(dim=0), int(member.any(dim=1).sum())
    share = counts.double() / max(1, entries)
    balance = experts * (share * p.sum(dim=0)).sum() / max(1, routed)
    outputs = [bounds(member.sum(dim=1)), padded(where[:, 1].to(torch.int32), -1), padded(gate[member], 0.0),
               padded(number[member].to(torch.int32), -1), bounds(counts), padded(by_expert[:, 1].to(torch.int32), -1),
               counts.to(torch.int32), lse, balance.reshape(1)]
    if case["mode"] == "train":
        dg = torch.zeros_like(p)
        dg[member] = s["grad_gate"].double().cpu()[:entries]
        inner = (gate * dg).sum(dim=1, keepdim=True)
        grad = gate * (dg - inner) if case["normalise"] else gate * dg - p * inner
        c = BALANCE * experts * share / max(1, routed)
        outputs.append(grad + p * (c - (p * c).sum(dim=1, keepdim=True)))
    return outputs


def _exact_experts(case, s):
    x, w, bounds, token = s["x"].double(), s["weight"].double(), s["bounds"].tolist(), s["token"].long()
    train, act = case["mode"] == "train", case["act"]
    parts = []
    for e in range(case["experts"]):
        rows = x[token[bounds[e]:bounds[e + 1]]]
        z = rows @ w[e].t().contiguous()
        if s["bias"] is not None:
            z = z + s["bias"][e].double()
        if act == "gelu":
            y = torch.nn.functional.gelu(z)
        elif act == "silu":
            y = torch.nn.functional.silu(z)
        else:
            y = torch.relu(z) if act == "relu" else z
        part = [y]
        if train:
            slope = torch.ones_like(z)
            if act == "gelu":
                slope = 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
            elif act == "silu":
                slope = torch.sigmoid(z) + y * torch.sigmoid(-z)
            elif act == "relu":
                slope = torch.where(z > 0, slope, torch.zeros_like(z))
            gz = s["grad_y"][bounds[e]:bounds[e + 1]].double() * slope
            part += [gz @ w[e], (gz.t().contiguous() @ rows)[None], gz.sum(dim=0)[None]]
        parts.append(part)
    outputs = [torch.cat(column) for column in zip(*parts)]
    return outputs[:3] if train and s["bias"] is None else outputs


def _exact_combine(case, s):
    pos, slot, gate, y = s["pos"].long(), s["slot"].long(), s["gate"].double(), s["y"].double()
    token = torch.repeat_interleave(torch.arange(case["tokens"], device=DEVICE), pos[1:] - pos[:-1])
    out = s["residual"].double() if s["residual"] is not None else torch.zeros((case["tokens"], case["outer"]), dtype=torch.float64, device=DEVICE)
    outputs = [out.index_add(0, token, y[slot] * gate[:, None])]
    if case["mode"] == "train":
        go = s["grad_out"].double()[token]
        grad_y = torch.zeros_like(y)
        grad_y[slot] = go * gate[:, None]
        outputs += [grad_y, (go * y[slot]).sum(dim=1)]
    return outputs


def exact(case, seed):
    s = _inputs(case, seed)
    return {"distill": _exact_distill, "route": _exact_route, "experts": _exact_experts, "combine": _exact_combine}[case["op"]](case, s)
