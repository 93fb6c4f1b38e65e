"""nacho_combine, nacho_combine_grad against the definition in 64 bits.

Tolerances: a sum of n products in 32 bits is within n 2^-24 of the sum of their magnitudes (n: entries and the
residual, or the columns), and results of 16 bits are rounded once (2^-8 of a bf16, 2^-11 of an f16, half the smallest
f16 step)."""
import numpy as np
import pytest
import torch

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
STEP = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def routing(rng, tokens, most, spare=0):
    """Rows of 0 .. most slots, all different; `spare` slots belong to no entry."""
    held = rng.integers(0, most + 1, tokens)
    pos = np.concatenate([[0], np.cumsum(held)]).astype(np.int32)
    slots = rng.permutation(pos[-1] + spare)[:pos[-1]]
    for t in range(tokens):
        slots[pos[t]:pos[t + 1]].sort()
    return pos, slots.astype(np.int32), rng.normal(0, 1, pos[-1]).astype(np.float32)


def dev(a):
    return torch.from_numpy(a).cuda()


def rows_of(rng, rows, cols, ld, dtype):
    return torch.from_numpy(rng.normal(0, 1, (rows, ld)).astype(np.float32)).to(dtype).cuda()[:, :cols]


def near(got, want, size, dtype, terms):
    g = got.float().cpu().numpy().astype(np.float64)
    return np.all(np.abs(g - want) <= STEP[dtype] * np.abs(want) + (terms + 4) * 2.0 ** -24 * size + 2.0 ** -25 * (dtype is torch.float16))


SHAPES = [(1, 1, 1), (3, 5, 2), (7, 64, 4), (2, 63, 9), (20, 100, 3), (5, 256, 2), (9, 1000, 4), (4, 1024, 8), (3, 4097, 5),
          (2, 4098, 4), (50, 2048, 1), (3, 33000, 3), (400, 48, 2)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,cols,most", SHAPES)
@pytest.mark.parametrize("kind", ["plain", "no_gate", "strided"])
def test_sums_and_gradients(tokens, cols, most, kind, dtype):
    rng = np.random.default_rng(tokens * 31 + cols)
    pos, slot, gate = routing(rng, tokens, most, 2)
    slots, ld = len(slot) + 2, cols + (8 if kind == "strided" else 0)
    y, residual, go = (rows_of(rng, n, cols, ld, dtype) for n in (slots, tokens, tokens))
    if kind == "no_gate":
        gate = np.ones_like(gate)
    g = None if kind == "no_gate" else dev(gate)
    token = np.repeat(np.arange(tokens), np.diff(pos))
    y64, r64, go64 = (t.float().cpu().numpy().astype(np.float64) for t in (y, residual, go))
    terms = y64[slot] * gate[:, None]
    want, size = np.zeros((tokens, cols)), np.zeros((tokens, cols))
    np.add.at(want, token, terms)
    np.add.at(size, token, np.abs(terms))
    P, S = dev(pos), dev(slot)
    assert near(nb.nacho_combine(P, S, y, gate=g), want, size, dtype, most)
    out = torch.full((tokens, ld), 7.0, dtype=dtype, device="cuda")
    nb.nacho_combine(P, S, y, gate=g, residual=residual, out=out[:, :cols])
    assert near(out[:, :cols], want + r64, size + np.abs(r64), dtype, most + 1) and bool((out[:, cols:] == 7.0).all())
    into = residual.clone()
    nb.nacho_combine(P, S, y, gate=g, residual=into, out=into)
    assert near(into, want + r64, size + np.abs(r64), dtype, most + 1)
    grad_y = torch.full((slots, ld), 7.0, dtype=dtype, device="cuda")
    _, grad_gate = nb.nacho_combine_grad(P, S, y, go, gate=g, grad_y=grad_y[:, :cols])
    want_y = np.full((slots, ld), 7.0)
    want_y[slot, :cols] = go64[token] * gate[:, None]
    assert near(grad_y, want_y, np.abs(want_y), dtype, 1)
    dots = go64[token] * y64[slot]
    assert near(grad_gate, dots.sum(1), np.abs(dots).sum(1), torch.float32, cols)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_places_behind_the_last_entry_are_not_read(dtype):
    rng = np.random.default_rng(2)
    pos, slot, gate = routing(rng, 6, 3)
    y = rows_of(rng, len(slot) + 4, 96, 96, dtype)
    y[len(slot):] = float("nan")
    full = nb.nacho_combine(dev(pos), dev(slot), y, gate=dev(gate))
    slot = np.concatenate([slot, -np.ones(5, np.int32)]).astype(np.int32)
    gate = np.concatenate([gate, np.full(5, np.nan, np.float32)]).astype(np.float32)
    assert torch.equal(full, nb.nacho_combine(dev(pos), dev(slot), y, gate=dev(gate)))
    assert bool(torch.isfinite(full.float()).all())
    empty = [t for t in range(6) if pos[t] == pos[t + 1]]
    assert not bool(full[empty].any())


def test_nothing_to_sum():
    y = torch.ones((3, 8), device="cuda")
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert nb.nacho_combine(pos, none, y).shape == (0, 8)
    pos = torch.zeros(5, dtype=torch.int32, device="cuda")
    assert not bool(nb.nacho_combine(pos, none, y).any())
    grad_y, grad_gate = nb.nacho_combine_grad(pos, none, y, torch.ones((4, 8), device="cuda"), grad_y=torch.full((3, 8), 2.0, device="cuda"))
    assert bool((grad_y == 2).all()) and grad_gate.numel() == 0


def test_offsets_past_two_to_the_31():
    """Rows of y whose offset passes 32 bits."""
    rows, cols = 70_000, 32_768                              # 2.3e9 elements, 4.6 GB
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    y[0], y[-1] = 2.0, 3.0
    pos = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    slot = torch.tensor([0, rows - 1], dtype=torch.int32, device="cuda")
    out = nb.nacho_combine(pos, slot, y, gate=torch.tensor([0.5, 4.0], device="cuda"))
    assert bool((out == 13).all())


def test_another_stream_and_the_same_bits_again():
    rng = np.random.default_rng(3)
    pos, slot, gate = (dev(a) for a in routing(rng, 500, 4))
    y, go = rows_of(rng, slot.numel(), 777, 777, torch.float16), rows_of(rng, 500, 777, 777, torch.float16)
    first = [nb.nacho_combine(pos, slot, y, gate=gate), *nb.nacho_combine_grad(pos, slot, y, go, gate=gate)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = [nb.nacho_combine(pos, slot, y, gate=gate), *nb.nacho_combine_grad(pos, slot, y, go, gate=gate)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_refusals():
    y = torch.ones((6, 16), device="cuda")
    pos = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda")
    slot = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        nb.nacho_combine(pos, slot, y.double())
    with pytest.raises(ValueError):
        nb.nacho_combine(pos.long(), slot, y)
    with pytest.raises(ValueError):
        nb.nacho_combine(pos, slot, y, gate=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        nb.nacho_combine(pos, slot, y, residual=torch.ones((3, 16), device="cuda"))
    with pytest.raises(nb.NachoError):
        nb.nacho_combine(pos, slot, y, out=y[:2])
    with pytest.raises(nb.NachoError):
        nb.nacho_combine(pos, slot, y, residual=y[2:4], out=y[3:5])
    with pytest.raises(nb.NachoError):
        nb.nacho_combine_grad(pos, slot, y, torch.ones((2, 16), device="cuda"), grad_y=y)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("words", [8, 9, 16, 17, 32, 33, 128, 129])
@pytest.mark.parametrize("odd", [0, 1])
def test_rows_on_both_sides_of_every_number_of_lanes(words, odd, dtype):
    """Rows of these numbers of words of 16 bytes, whole or with a last one that is not."""
    rng = np.random.default_rng(words)
    cols, tokens, most = words * (16 // torch.empty(0, dtype=dtype).element_size()) - odd, 37, 5
    pos, slot, gate = routing(rng, tokens, most)
    y, residual, go = (rows_of(rng, n, cols, cols, dtype) for n in (len(slot), tokens, tokens))
    token = np.repeat(np.arange(tokens), np.diff(pos))
    y64, r64, go64 = (t.float().cpu().numpy().astype(np.float64) for t in (y, residual, go))
    want, size = r64.copy(), np.abs(r64)
    np.add.at(want, token, y64[slot] * gate[:, None])
    np.add.at(size, token, np.abs(y64[slot] * gate[:, None]))
    assert near(nb.nacho_combine(dev(pos), dev(slot), y, gate=dev(gate), residual=residual), want, size, dtype, most + 1)
    grad_y, grad_gate = nb.nacho_combine_grad(dev(pos), dev(slot), y, go, gate=dev(gate))
    want_y = np.empty((len(slot), cols))
    want_y[slot] = go64[token] * gate[:, None]
    assert near(grad_y, want_y, np.abs(want_y), dtype, 1)
    dots = go64[token] * y64[slot]
    assert near(grad_gate, dots.sum(1), np.abs(dots).sum(1), torch.float32, cols)
