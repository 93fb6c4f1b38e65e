"""nacho_keep8, nacho_restore8 against the definition, bit by bit; nacho_experts_keep8 and nacho_experts_keep8_grad against it and against
the operators that keep their rows in the type.

Codes are whole numbers and steps powers of two, so rows of any type have one right answer.  Where the rows are sums of n products
held in 32 bits (within (n + 8) 2^-24 of the sum of their magnitudes), a kept row is within half a step and that error of them, one
step where it has more than 127 of them."""
import math

import numpy as np
import pytest
import torch

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def definition(x):
    """Codes and exponents of rows, by the definition, in 64 bits."""
    v = x.cpu().double().numpy()
    rows, cols = v.shape
    blocks = -(-cols // 32)
    codes, exponent = np.zeros((rows, cols), dtype=np.int8), np.zeros((rows, blocks), dtype=np.uint8)
    for b in range(blocks):
        part = v[:, b * 32:(b + 1) * 32]
        with np.errstate(invalid="ignore"):
            most = np.abs(part).max(axis=1)
        for r in range(rows):
            if not np.isfinite(most[r]):
                exponent[r, b] = 255
                continue
            e = max(math.frexp(most[r])[1] - 1 + 121, 0) if most[r] > 0 else 0
            exponent[r, b] = e
            codes[r, b * 32:(b + 1) * 32] = np.clip(np.rint(part[r] / 2.0 ** (e - 127)), -127, 127)
    return torch.from_numpy(codes), torch.from_numpy(exponent)


def values(codes, exponent):
    step = torch.pow(2.0, exponent.cpu().double() - 127)
    step[exponent.cpu() == 255] = math.nan
    return codes.cpu().double() * step.repeat_interleave(32, dim=1)[:, :codes.shape[1]]


def check(x):
    kept = nb.nacho_keep8(x)
    codes, exponent = definition(x)
    assert torch.equal(kept.exponent.cpu(), exponent) and torch.equal(kept.codes.cpu(), codes)
    want = values(codes, exponent)
    for dtype in TYPES:
        got = nb.nacho_restore8(kept, dtype).cpu()
        assert got.dtype is dtype and torch.equal(got.isnan(), want.isnan())
        # (a value past the type's range is an infinity there)
        assert torch.equal(got.masked_fill(got.isnan(), 7.0), want.masked_fill(want.isnan(), 7.0).to(dtype))
    return kept


def rows_of(seed, rows, cols, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g).float())
    return x.to(dtype)


SIZES = [(1, 1), (1, 16), (3, 31), (5, 32), (7, 33), (2, 48), (4, 100), (65, 1000), (1000, 3), (300, 17), (9, 4096), (2, 40_001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_every_code(rows, cols, dtype):
    x = rows_of(rows + cols, rows, cols, dtype)
    kept = check(x.cuda())
    step = torch.pow(2.0, kept.exponent.cpu().double() - 127).repeat_interleave(32, dim=1)[:, :cols]
    off = (values(kept.codes, kept.exponent) - x.double()).abs() / step
    assert bool((off <= torch.where(x.double().abs() / step > 127.5, 1.0, 0.5)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(1, 0), (16, 0), (8, 3), (0, 1)])
def test_rows_apart_and_anywhere(dtype, pad, shift):
    """Rows with gaps that start at any element; what lies between them is left."""
    rows, cols = 13, 75
    x = rows_of(pad, rows, cols, dtype)
    place = lambda dtype, fill, width: torch.full((shift + rows * (width + pad),), fill, dtype=dtype, device="cuda")
    view = lambda whole, width: whole[shift:].view(rows, width + pad)[:, :width]
    wide = place(dtype, 5.0, cols)
    view(wide, cols).copy_(x)
    codes, exponent, out = place(torch.int8, 99, cols), place(torch.uint8, 77, 3), place(dtype, 3.0, cols)
    kept = nb.Kept8(view(codes, cols), view(exponent, 3))
    assert nb.nacho_keep8(view(wide, cols), out=kept) is kept
    nb.nacho_restore8(kept, out=view(out, cols))
    c, e = definition(x)
    assert torch.equal(kept.codes.cpu(), c) and torch.equal(kept.exponent.cpu(), e) and torch.equal(view(out, cols).cpu().double(), values(c, e).to(dtype).double())
    for whole, fill, width in ((codes, 99, cols), (exponent, 77, 3), (out, 3.0, cols)):
        assert bool((whole[:shift] == fill).all())
        if pad:
            assert bool((whole[shift:].view(rows, width + pad)[:, width:] == fill).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_values_at_the_edges(dtype):
    """Ties, zeros, the largest and smallest numbers of the type, infinities and NaN."""
    x = torch.zeros((12, 96), dtype=dtype)
    x[0, :32] = torch.tensor([64.0] + [i / 2 for i in range(-15, 16)]).to(dtype)        # halves: ties to even
    x[1, :4] = torch.tensor([127.0, 127.49, -127.9, 126.5]).to(dtype)
    x[2, 40] = torch.finfo(dtype).max
    x[2, 41] = torch.finfo(dtype).min
    x[3, 0] = torch.finfo(dtype).tiny
    x[3, 33] = torch.finfo(dtype).tiny / 4                                              # (smaller than normal numbers)
    x[4, 5], x[5, 70], x[6, 95] = math.nan, math.inf, -math.inf
    x[4, 64:] = 1.0
    x[7] = -0.0
    x[8] = 1.0
    x[9] = torch.linspace(-1, 1, 96).to(dtype)
    x[10, 0], x[10, 1] = 1.0, 2.0 ** -8
    x[11] = torch.linspace(0.0, 2.0 ** -13, 96).to(dtype)
    check(x.cuda())
    if dtype is torch.float32:
        tiny = torch.zeros((3, 64))
        tiny[0, 0], tiny[1, :2], tiny[2, 40] = 2.0 ** -149, torch.tensor([2.0 ** -121, 2.0 ** -128]), 2.0 ** -127
        check(tiny.cuda())


def test_no_row_and_no_column():
    for shape in ((0, 40), (7, 0)):
        kept = nb.nacho_keep8(torch.zeros(shape, device="cuda"))
        assert kept.shape == shape and nb.nacho_restore8(kept, torch.float16).shape == shape


def test_more_than_2_31_elements():
    rows, cols = 70_000, 32_768
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in (0, 1, 65_535, 65_536, rows - 1):
        x[r] = rows_of(r, 1, cols, torch.bfloat16)[0]
    kept = nb.nacho_keep8(x)
    back = nb.nacho_restore8(kept, torch.bfloat16)
    for r in (0, 1, 65_535, 65_536, rows - 1):
        codes, exponent = definition(x[r:r + 1])
        assert torch.equal(kept.codes[r:r + 1].cpu(), codes) and torch.equal(kept.exponent[r:r + 1].cpu(), exponent)
        assert torch.equal(back[r].cpu().double(), values(codes, exponent)[0])
    assert int(back[2:65_535].count_nonzero()) == 0


def layer(seed, counts, tokens, inner, outer, dtype, bias, pad=0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g)
    apart = lambda t: torch.cat([t, torch.full((*t.shape[:-1], pad), float("nan"))], dim=-1).to(dtype).cuda()[..., :t.shape[-1]]
    slots = sum(counts)
    return dict(x=apart(rand(tokens, inner)), w=apart(rand(len(counts), outer, inner) * inner ** -0.5), gy=apart(rand(slots, outer)),
                bias=rand(len(counts), outer).to(dtype).cuda() if bias else None, slots=slots,
                bounds=torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda"),
                token=torch.randint(0, tokens, (slots,), generator=g, dtype=torch.int32).cuda())


LAYERS = [([1], 1, 1, 1), ([3], 5, 8, 8), ([0, 2, 0], 4, 16, 24), ([5, 1, 130], 40, 32, 64), ([17, 16, 15], 9, 40, 136), ([70, 300], 64, 33, 77),
          ([260, 10], 100, 128, 256), ([300] * 4, 500, 64, 512), ([600, 520], 700, 24, 40_000 // 4)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", LAYERS)
def test_a_layer_that_keeps_its_rows(case, dtype):
    """Forward: the same results as without keeping, kept rows next to the sums.  Back: the bits that the operator which takes rows of
    the type gives for the rows that the codes stand for (of 16 bits these are exact)."""
    counts, tokens, inner, outer = case
    seed = inner + outer
    act = ["none", "relu", "gelu", "silu"][seed % 4] if outer > 1 else "gelu"
    d = layer(seed, counts, tokens, inner, outer, dtype, seed % 2 == 0, pad=seed % 3)
    room = d["slots"] + 2
    pre = nb.Kept8(torch.full((room, outer), 99, dtype=torch.int8, device="cuda"), torch.full((room, -(-outer // 32)), 77, dtype=torch.uint8, device="cuda"))
    more = dict(token=torch.cat([d["token"], d["token"].new_zeros(2)]), act=act)
    y = torch.full((room, outer), 7.0, dtype=dtype, device="cuda")
    nb.nacho_experts(d["x"], d["w"], d["bounds"], bias=d["bias"], y=y, pre=pre, **more)
    plain = torch.full((room, outer), 7.0, dtype=dtype, device="cuda")
    rows = torch.full((room, outer), 7.0, dtype=dtype, device="cuda")
    nb.nacho_experts(d["x"], d["w"], d["bounds"], bias=d["bias"], y=plain, pre=rows, **more)
    slots = d["slots"]
    assert torch.equal(y, plain) and bool((pre.codes[slots:] == 99).all()) and bool((pre.exponent[slots:] == 77).all())
    if dtype is torch.float32:
        again = nb.nacho_keep8(rows[:slots])
        assert torch.equal(pre.codes[:slots], again.codes) and torch.equal(pre.exponent[:slots], again.exponent)
    bounds = d["bounds"].tolist()
    for e in range(len(counts)):
        a, b = bounds[e], bounds[e + 1]
        xs, w = d["x"][d["token"][a:b].long()].cpu().double(), d["w"][e].cpu().double()
        z, size = xs @ w.T, xs.abs() @ w.abs().T
        if d["bias"] is not None:
            z, size = z + d["bias"][e].cpu().double(), size + d["bias"][e].cpu().double().abs()
        step = torch.pow(2.0, pre.exponent[a:b].cpu().double() - 127).repeat_interleave(32, dim=1)[:, :outer]
        off = (values(pre.codes[a:b], pre.exponent[a:b]) - z).abs() - (inner + 8) * 2.0 ** -24 * size
        assert bool((off <= step * torch.where(pre.codes[a:b].cpu().abs() == 127, 1.0, 0.5)).all())
    gy = torch.cat([d["gy"], torch.full((2, outer), float("nan"), dtype=dtype, device="cuda")])
    kept_x = nb.nacho_keep8(d["x"])
    x = nb.nacho_restore8(kept_x, dtype)
    z = nb.nacho_restore8(pre, dtype)
    back = dict(token=more["token"], act=act)
    for kx, kp in ((True, True), (True, False), (False, True)):
        gb, want_gb = (torch.full((len(counts), outer), 7.0, dtype=dtype, device="cuda") for _ in range(2))
        got = nb.nacho_experts_grad(gy, kept_x if kx else x, d["w"], d["bounds"], pre=pre if kp else z, grad_bias=gb, **back)
        want = nb.nacho_experts_grad(gy, x, d["w"], d["bounds"], pre=z, grad_bias=want_gb, **back)
        assert torch.equal(got[0][:slots], want[0][:slots]) and torch.equal(got[1], want[1]) and torch.equal(gb, want_gb), (kx, kp)
    gx, none = nb.nacho_experts_grad(gy, kept_x, d["w"], d["bounds"], pre=pre, grad_weight=False, **back)
    assert none is None and torch.equal(gx[:slots], got[0][:slots])


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_gradients_of_kept_rows_against_the_definition(act):
    """In 32 bits, from the values that the codes stand for, in 64.  (A slope has an error of a few 2^-24; a product's terms are sums
    as in the forward call.)"""
    d = layer(3, [40, 7, 0, 19], 30, 48, 70, torch.float32, False)
    pre, x = nb.Kept8.empty(d["slots"], 70, "cuda"), nb.nacho_keep8(d["x"])
    nb.nacho_experts(d["x"], d["w"], d["bounds"], token=d["token"], act=act, pre=pre)
    gb = torch.empty((4, 70), device="cuda")
    gx, gw = nb.nacho_experts_grad(d["gy"], x, d["w"], d["bounds"], token=d["token"], act=act, pre=pre, grad_bias=gb)
    z, xs = values(pre.codes, pre.exponent).requires_grad_(), values(x.codes, x.exponent)[d["token"].long().cpu()]
    {"gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu, "relu": torch.relu}[act](z).backward(d["gy"].cpu().double())
    w, bounds = d["w"].cpu().double(), d["bounds"].tolist()
    for e in range(4):
        a, b = bounds[e], bounds[e + 1]
        g, size = z.grad[a:b], d["gy"][a:b].cpu().double().abs() * 1.2
        for got, want, room in ((gx[a:b], g @ w[e], size @ w[e].abs() * (70 + 16)), (gw[e], g.T @ xs[a:b], size.T @ xs[a:b].abs() * (b - a + 16)),
                                (gb[e], g.sum(0), size.sum(0) * (b - a + 16))):
            assert bool(((got.cpu().double() - want).abs() <= room * 2.0 ** -24).all())


def test_rows_with_a_nan_are_restored_as_nan():
    """(32 columns together, and no others)"""
    x = torch.ones((3, 100), device="cuda")
    x[1, 40] = math.inf
    back = nb.nacho_restore8(nb.nacho_keep8(x), torch.float16)
    assert bool(back[1, 32:64].isnan().all()) and int(back.isnan().sum()) == 32


def test_under_captured_graphs():
    d = layer(5, [90, 30, 45], 60, 64, 96, torch.bfloat16, True)

    def work():
        pre = nb.Kept8.empty(d["slots"], 96, "cuda")
        y = nb.nacho_experts(d["x"], d["w"], d["bounds"], token=d["token"], bias=d["bias"], act="gelu", pre=pre)
        x = nb.nacho_keep8(d["x"])
        return [y, pre.codes, pre.exponent, x.codes, x.exponent, nb.nacho_restore8(x, torch.bfloat16),
                *nb.nacho_experts_grad(d["gy"], x, d["w"], d["bounds"], token=d["token"], act="gelu", pre=pre)]

    work()
    torch.cuda.synchronize()
    graphs, results = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            results.append(work())
    for seed in range(4):
        torch.manual_seed(seed)
        d["x"].normal_()
        d["gy"].normal_()
        graphs[0].replay()
        torch.cuda.synchronize()
        eager = work()
        graphs[1].replay()
        torch.cuda.synchronize()
        for result in results:
            assert all(torch.equal(a, b) for a, b in zip(result, eager))
