"""nacho_experts_step against the definition in 64 bits.

Tolerances: a sum of n products held in 32 bits is within (n + 8) 2^-24 of the sum of their magnitudes; an activation passes on
1.2 of its argument's error and adds a few 2^-24 of its argument; the rows between the products are rounded to the type, and the
result once (2^-8 of a bf16, 2^-11 of an f16, half the smallest f16 step).  A gate is off by 2^-22 of its logit's distance from the
largest one (the argument of its exponential, an instruction of 2^-22), and by the sum of n_experts such numbers: 2^-17 for logits
that differ by less than 16."""
import math

import pytest
import torch

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ACTS = ["none", "relu", "gelu", "silu"]


def act64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    return z * torch.sigmoid(z) if act == "silu" else z


def strided(t, pad):
    """The same values in rows `pad` elements further apart, the gaps filled with NaN."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + pad), float("nan"), dtype=t.dtype)
    wide[..., :t.shape[-1]] = t
    return wide.cuda()[..., :t.shape[-1]]


def problem(seed, tokens, experts, inner, hidden, outer, dtype, gated=False, bias=False, residual=False, keep=False):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g)
    d = dict(x=rand(tokens, inner), logits=rand(tokens, experts), up=rand(experts, hidden, inner) * inner ** -0.5,
             down=rand(experts, outer, hidden) * hidden ** -0.5, gate=rand(experts, hidden, inner) * inner ** -0.5 if gated else None,
             up_bias=rand(experts, hidden) if bias else None, gate_bias=rand(experts, hidden) if bias and gated else None,
             down_bias=rand(experts, outer) if bias else None, residual=rand(tokens, outer) if residual else None)
    d = {n: None if t is None else t.to(dtype) for n, t in d.items()}
    d["keep"] = torch.rand(tokens, generator=g) < 0.7 if keep else None
    return d


def routed(d, top_k, normalise):
    """(token, expert, gate) of every choice, by the definition."""
    z = d["logits"].double()
    for t in range(z.shape[0]):
        if d["keep"] is not None and not d["keep"][t]:
            continue
        row = z[t]
        order = sorted((e for e in range(z.shape[1]) if row[e] > -math.inf), key=lambda e: (-row[e], e))[:top_k]
        p = torch.softmax(row, 0)
        whole = p[order].sum() if normalise else 1.0
        for e in order:
            yield t, e, (p[e] / whole).item()


def reference(d, top_k, normalise, act, dtype):
    """The result in 64 bits, and by how much it may be off."""
    w = {n: None if t is None or n == "keep" else t.double() for n, t in d.items()}
    tokens, outer = d["x"].shape[0], d["down"].shape[1]
    inner, hidden = d["x"].shape[1], d["up"].shape[1]
    out = w["residual"].clone() if w["residual"] is not None else torch.zeros((tokens, outer), dtype=torch.float64)
    sizes, room = out.abs(), torch.zeros_like(out)
    half, tiny = (0.0 if dtype is torch.float32 else HALF[dtype]), 2.0 ** -25 * (dtype is torch.float16)
    f32 = lambda n: (n + 8) * 2.0 ** -24
    for t, e, g in routed(d, top_k, normalise):
        def product(name):
            z, size = w[name][e] @ w["x"][t], w[name][e].abs() @ w["x"][t].abs()
            if w[name + "_bias"] is not None:
                z, size = z + w[name + "_bias"][e], size + w[name + "_bias"][e].abs()
            return z, size
        z, size = product("up")
        if w["gate"] is not None:
            a, asize = product("gate")
            h = act64(a, act) * z
            off = f32(inner) * ((1.2 * asize + 4 * a.abs()) * (z.abs() + f32(inner) * size) + act64(a, act).abs() * size)
        else:
            h = act64(z, act)
            off = f32(inner) * (1.2 * size + 4 * z.abs())
        off = off + half * (h.abs() + off) + tiny
        y, ysize = w["down"][e] @ h, w["down"][e].abs() @ h.abs()
        if w["down_bias"] is not None:
            y, ysize = y + w["down_bias"][e], ysize + w["down_bias"][e].abs()
        out[t] += g * y
        sizes[t] += g * ysize
        room[t] += g * (w["down"][e].abs() @ off) + 2.0 ** -17 * g * ysize
    room = room + f32(hidden * top_k + 2 * top_k) * sizes
    return out, room + HALF[dtype] * (out.abs() + room) + tiny


def on_gpu(d, pad=0):
    return {n: None if t is None else strided(t, pad) if pad and n not in ("keep",) else t.cuda() for n, t in d.items()}


def run(d, top_k, act, normalise, pad=0, **more):
    g = on_gpu(d, pad)
    return nb.nacho_experts_step(g["x"], g["logits"], top_k, g["up"], g["down"], gate=g["gate"], up_bias=g["up_bias"], gate_bias=g["gate_bias"],
                                 down_bias=g["down_bias"], act=act, normalise=normalise, keep=g["keep"], residual=g["residual"], **more)


def check(d, top_k, act, normalise, dtype, pad=0):
    tokens, outer = d["x"].shape[0], d["down"].shape[1]
    wide = torch.full((tokens + 1, outer + pad), 7.0, dtype=dtype, device="cuda")
    got = run(d, top_k, act, normalise, pad, out=wide[:tokens, :outer])
    want, room = reference(d, top_k, normalise, act, dtype)
    wrong = ((got.cpu().double() - want).abs() - room).max()
    assert bool(((got.cpu().double() - want).abs() <= room).all()), float(wrong)
    assert bool((wide[tokens:] == 7.0).all()) and bool((wide[:, outer:] == 7.0).all())
    assert torch.equal(got, run(d, top_k, act, normalise, pad))


SIZES = [(1, 1, 1, 1, 1, 1), (1, 4, 2, 8, 16, 24), (1, 64, 8, 256, 64, 128), (3, 5, 3, 7, 9, 5), (2, 3, 2, 1, 40, 17), (4, 3, 2, 40, 3, 50), (16, 8, 2, 64, 96, 48),
         (17, 8, 2, 64, 96, 40), (64, 6, 6, 72, 130, 33), (64, 70, 4, 33, 65, 31), (64, 2, 1, 128, 64, 64), (33, 1, 1, 48, 32, 16), (5, 1024, 32, 16, 24, 20),
         (2, 200, 8, 264, 520, 264), (9, 65, 5, 1025, 257, 129), (1, 8, 1, 2048, 2048, 512),
         (3, 40, 32, 24, 40, 24), (64, 33, 32, 24, 16, 24), (2, 300, 32, 24, 40, 24), (40, 1, 1, 512, 264, 48)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("gated", [False, True])
def test_against_the_definition(sizes, dtype, gated):
    tokens, experts, top_k, inner, hidden, outer = sizes
    seed = tokens * 7 + experts + hidden
    d = problem(seed, tokens, experts, inner, hidden, outer, dtype, gated=gated, bias=seed % 2 == 0, residual=seed % 3 == 0, keep=seed % 5 == 0)
    check(d, top_k, ACTS[seed % 4], seed % 2 == 1, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("act", ACTS)
def test_rows_apart(dtype, pad, act):
    """Rows, matrices and biases with gaps (of NaN) between them."""
    d = problem(pad, 7, 6, 48, 56, 40, dtype, gated=pad == 3, bias=True, residual=True, keep=True)
    check(d, 2, act, True, dtype, pad)


# Tiles of 16 rows of the experts that tokens can choose, from 2048 on: a wavefront has one at a time, with all of k.  Rows of words,
# rows that start anywhere, rows shorter than 16 bytes; one stretch of k and several with a last one that is not whole; experts of more
# than 16 tokens (2048 choices of 70 experts, 64 of one).
MANY_ITEMS = [(64, 128, 8, 40, 256, 24), (64, 128, 8, 200, 256, 24), (64, 128, 8, 203, 261, 19), (64, 128, 8, 3, 260, 17), (64, 70, 32, 72, 520, 24),
              (64, 70, 32, 75, 520, 21), (9, 300, 32, 136, 128, 40), (64, 1, 1, 72, 33_000, 9)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("sizes", MANY_ITEMS)
def test_many_items(sizes, gated, dtype):
    tokens, experts, top_k, inner, hidden, outer = sizes
    assert min(tokens * top_k, experts) * -(-hidden // 16) >= 2048
    d = problem(sum(sizes), tokens, experts, inner, hidden, outer, dtype, gated=gated, bias=True, residual=gated, keep=not gated)
    act = ACTS[sum(sizes) % 4]
    check(d, top_k, act, True, dtype)
    check(d, top_k, act, False, dtype, pad=8 if inner % 8 == 0 else 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [(7, 6, 2, 72, 56, 40), (64, 128, 8, 135, 256, 24)])
@pytest.mark.parametrize("name", ["x", "up", "gate", "down"])
def test_arrays_that_start_at_an_odd_element(name, sizes, dtype):
    """16-bit arrays whose first row starts between two words of 4 bytes, which are read element by element."""
    tokens, experts, top_k, inner, hidden, outer = sizes
    d = problem(sum(sizes), tokens, experts, inner, hidden, outer, dtype, gated=True)
    g = on_gpu(d)
    room = torch.full((g[name].numel() + 2,), float("nan"), dtype=dtype, device="cuda")
    room[1:-1] = g[name].flatten()
    g[name] = room[1:-1].view(g[name].shape)
    assert g[name].data_ptr() % 4 == 2
    got = nb.nacho_experts_step(g["x"], g["logits"], top_k, g["up"], g["down"], gate=g["gate"], normalise=True)
    want, off = reference(d, top_k, True, "silu", dtype)
    assert bool(((got.cpu().double() - want).abs() <= off).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_and_experts_that_are_closed(dtype):
    """Equal logits go to the lowest index; -inf and NaN are never chosen, and a token may choose fewer or none."""
    d = problem(3, 6, 9, 24, 32, 40, dtype, residual=True)
    z = d["logits"]
    z[0] = 1.0
    z[1] = torch.tensor([0, 2, 2, 2, 1, 2, 0, 0, 2], dtype=dtype)
    z[2] = -math.inf
    z[3] = -math.inf
    z[3, 5] = 0.25
    z[4, 2:] = -math.inf
    check(d, 4, "gelu", True, dtype)
    check(d, 4, "gelu", False, dtype)
    assert torch.equal(run(d, 4, "gelu", True)[2].cpu(), d["residual"][2])


def test_a_nan_among_the_logits():
    """It is not chosen, and makes that token's gates, and no others, NaN."""
    d = problem(5, 4, 8, 16, 16, 24, torch.float32)
    clean = run(d, 2, "silu", False)
    d["logits"][1, 3] = math.nan
    got = run(d, 2, "silu", False)
    assert bool(got[1].isnan().all()) and torch.equal(got[[0, 2, 3]], clean[[0, 2, 3]])


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_read(dtype):
    """Weights of experts that nobody chose, and rows of tokens that are left out, may hold anything."""
    d = problem(6, 5, 12, 40, 48, 32, dtype, gated=True, bias=True, residual=True)
    d["keep"] = torch.tensor([True, True, False, True, False])
    clean = run(d, 2, "silu", True)
    chosen = {e for _, e, _ in routed(d, 2, True)}
    for e in set(range(12)) - chosen:
        for n in ("up", "gate", "down", "up_bias", "gate_bias", "down_bias"):
            d[n][e] = math.nan
    for t in (2, 4):
        d["x"][t] = math.nan
        d["logits"][t] = math.nan
    assert torch.equal(run(d, 2, "silu", True), clean)
    assert torch.equal(clean[[2, 4]].cpu(), d["residual"][[2, 4]])


def test_an_infinite_weight_stays_with_the_tokens_that_read_it():
    d = problem(8, 20, 4, 32, 32, 32, torch.float32)
    clean = run(d, 1, "relu", False)
    takers = sorted({t for t, e, _ in routed(d, 1, False) if e == 2})
    others = [t for t in range(20) if t not in takers]
    d["up"][2, 5] = math.nan
    d["down"][2, 7, 9] = math.inf
    got = run(d, 1, "relu", False)
    assert takers and others and torch.equal(got[others], clean[others]) and bool(got[takers].isnan().any())


def test_in_place_of_the_residual():
    d = problem(9, 10, 6, 64, 48, 72, torch.bfloat16, residual=True)
    want = run(d, 2, "silu", True)
    d["residual"] = d["residual"].cuda()
    got = nb.nacho_experts_step(d["x"].cuda(), d["logits"].cuda(), 2, d["up"].cuda(), d["down"].cuda(), act="silu", normalise=True,
                                residual=d["residual"], out=d["residual"])
    assert got is d["residual"] and torch.equal(got, want)


def test_no_token_takes_part():
    d = problem(9, 4, 6, 64, 48, 72, torch.bfloat16, bias=True, residual=True)
    d["keep"] = torch.zeros(4, dtype=torch.bool)
    assert torch.equal(run(d, 2, "silu", True).cpu(), d["residual"])
    d["residual"] = None
    assert int(run(d, 2, "silu", False).count_nonzero()) == 0


def test_more_than_2_31_weights():
    """The last experts' weights lie more than 2^32 bytes behind the first ones'."""
    experts, hidden, inner, outer = 300, 2048, 4096, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    up = torch.zeros((experts, hidden, inner), dtype=torch.bfloat16, device="cuda")
    d = problem(1, 2, experts, inner, 8, outer, torch.bfloat16)
    d["logits"][:, [3, 297, 299]] = 9.0
    for e in (3, 297, 299):
        up[e] = torch.randn((hidden, inner), generator=g, device="cuda") * inner ** -0.5
    down = (torch.randn((experts, outer, hidden), generator=g, device="cuda") * hidden ** -0.5).to(torch.bfloat16)
    got = nb.nacho_experts_step(d["x"].cuda(), d["logits"].cuda(), 3, up, down, act="silu", normalise=True)
    small = {**d, "up": up[[3, 297, 299]].cpu(), "down": down[[3, 297, 299]].cpu(), "logits": d["logits"][:, [3, 297, 299]]}
    want, room = reference(small, 3, True, "silu", torch.bfloat16)
    assert bool(((got.cpu().double() - want).abs() <= room).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(1, 1, 1, 1, 1, 1), (1, 64, 8, 256, 64, 128), (5, 1024, 32, 16, 24, 20), (9, 65, 5, 1025, 257, 129), (64, 6, 6, 72, 130, 33), (64, 128, 8, 40, 256, 24)])
def test_workspaces_are_enough(sizes, dtype):
    """A call with a workspace of the bytes that were asked for writes nothing behind it, and gives what one with its own gives."""
    tokens, experts, top_k, inner, hidden, outer = sizes
    d = problem(sum(sizes), tokens, experts, inner, hidden, outer, dtype, bias=True, residual=True)
    asked = []
    rooms = nb._room_for
    try:
        nb._room_for = lambda call, c, ws, device: asked.append(rooms(call, c, None, device)[1]) or rooms(call, c, ws, device)
        want = run(d, top_k, "silu", True)
    finally:
        nb._room_for = rooms
    room = torch.full((asked[0] + (1 << 16),), 0x5a, dtype=torch.uint8, device="cuda")
    got = run(d, top_k, "silu", True, ws=room[:asked[0]])
    assert torch.equal(got, want) and bool((room[asked[0]:] == 0x5a).all())


def test_no_token():
    d = problem(9, 1, 6, 64, 48, 72, torch.float32)
    g = on_gpu(d)
    assert nb.nacho_experts_step(g["x"][:0], g["logits"][:0], 2, g["up"], g["down"]).shape == (0, 72)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [1, 13, 64])
def test_the_operators_one_by_one(dtype, tokens):
    """Routing, both products and the sum give the same but for the rounding of the second product's rows."""
    d = problem(tokens, tokens, 10, 96, 160, 80, dtype, bias=True, residual=True)
    g = on_gpu(d)
    got = run(d, 3, "gelu", True)
    r = nb.nacho_route(g["logits"], 3, normalise=True)
    h = nb.nacho_experts(g["x"], g["up"], r.expert_pos, token=r.token, bias=g["up_bias"], act="gelu")
    y = nb.nacho_experts(h, g["down"], r.expert_pos, bias=g["down_bias"])
    plain = nb.nacho_combine(r.pos, r.slot, y, gate=r.gate, residual=g["residual"])
    want, room = reference(d, 3, True, "gelu", dtype)
    # (the rows of the second product: half a step of each, weighted)
    extra = torch.zeros_like(room)
    for t, e, gate in routed(d, 3, True):
        hidden = act64(d["up"][e].double() @ d["x"][t].double() + d["up_bias"][e].double(), "gelu")
        extra[t] += gate * HALF[dtype] * (d["down"][e].double() @ hidden + d["down_bias"][e].double()).abs() * 1.01 + 2.0 ** -25
    assert bool(((got.cpu().double() - plain.cpu().double()).abs() <= 2 * room + extra).all())


def test_on_another_stream_and_under_a_captured_graph():
    d = problem(2, 12, 16, 128, 96, 640, torch.bfloat16, gated=True, residual=True)
    g = on_gpu(d)
    work = lambda: nb.nacho_experts_step(g["x"], g["logits"], 4, g["up"], g["down"], gate=g["gate"], residual=g["residual"], normalise=True)
    want = work()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = work()
    side.synchronize()
    assert torch.equal(got, want)
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        one = work()
    with torch.cuda.graph(second):
        two = work()
    for seed in range(4):
        torch.manual_seed(seed)
        g["x"].normal_()
        g["logits"].normal_()
        first.replay()
        torch.cuda.synchronize()
        eager = work()
        second.replay()
        torch.cuda.synchronize()
        assert torch.equal(one, eager) and torch.equal(two, eager)
