"""nacho_xent, nacho_xent_grad against the definition in 64 bits.

Tolerances: a logit, a sum of n products held in 32 bits, is within dz = (n + 8) 2^-24 of the sum of their magnitudes.  An lse is off
by the largest dz of its row, 2^-21 for the exponentials (an argument and an instruction of 2^-22 each where a share is not
negligible), 2^-24 for every step of a sum (64 in a tile, then the tiles of a row), and two roundings of itself.  Of the gradient's
g = w (q - [label]) the share q is off by dz, the lse's error, 2^-21 + |z - lse| 2^-22 of itself; g is then rounded to the type (f16:
at a scale that leaves 2^-38 of the largest weight).  A share below 2^-126, the smallest normal number of 32 bits, is 0: the
exponential's instruction makes nothing smaller, so q is off by as much.  Products of g are sums as above; results are rounded to the type once."""
import pytest
import torch

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F32 = 2.0 ** -24


def apart(t, pad):
    """The same values in rows `pad` elements further apart, the gaps filled with NaN."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def problem(seed, rows, vocabulary, inner, dtype, weighted=True, masked=0.0, size=2.0, pad=0, label=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    labels = torch.randint(0, vocabulary, (rows,), generator=g, device="cuda", dtype=label)
    labels[torch.rand(rows, generator=g, device="cuda") < masked] = -100
    d = dict(x=new(rows, inner).to(dtype), head=(new(vocabulary, inner) * size * inner ** -0.5).to(dtype), label=labels,
             weight=0.25 + torch.rand(rows, generator=g, device="cuda") if weighted else None)
    if pad:
        d["x"], d["head"] = apart(d["x"], pad), apart(d["head"], pad)
    return d


def definition(d, dtype):
    """Results in 64 bits and by how much they may be off: {name: (value, room)}."""
    x, w = d["x"].double(), d["head"].double()
    rows, vocabulary, inner = x.shape[0], w.shape[0], x.shape[1]
    weight = d["weight"].double() if d["weight"] is not None else torch.ones(rows, dtype=torch.float64, device="cuda")
    held = (d["label"] >= 0) & (d["label"] < vocabulary) & (weight != 0)
    x, weight = torch.where(held[:, None], x, torch.zeros_like(x)), torch.where(held, weight, torch.zeros_like(weight))
    at = torch.where(held, d["label"], torch.zeros_like(d["label"])).long()[:, None]
    z, dz = x @ w.t().contiguous(), (inner + 8) * F32 * (x.abs() @ w.abs().t().contiguous())
    lse = torch.logsumexp(z, dim=1)
    d_lse = dz.max(dim=1)[0] + 2.0 ** -21 + (64 + vocabulary / 2048) * F32 + 2 * F32 * lse.abs()
    zl, dzl = torch.gather(z, 1, at)[:, 0], torch.gather(dz, 1, at)[:, 0]
    out = dict(lse=(torch.where(held, lse, 0.0), d_lse),
               loss=(weight * (lse - zl), weight.abs() * (d_lse + dzl + 4 * F32 * (lse - zl).abs() + 2 * F32 * (lse.abs() + zl.abs()))))
    q = torch.exp(z - lse[:, None])
    g = q.scatter_add(1, at, -torch.ones_like(zl)[:, None]) * weight[:, None]
    half = 0.0 if dtype is torch.float32 else HALF[dtype]
    dg = weight.abs()[:, None] * (q * (dz + d_lse[:, None] + 2.0 ** -21 + 2.0 ** -22 * (z - lse[:, None]).abs()) + 2 * F32 * g.abs() + 2 * F32 * q + 2.0 ** -126)
    dg = dg + half * (g.abs() + dg) + (2.0 ** -38 * weight.abs().max() * held[:, None] if dtype is torch.float16 and rows else 0.0)
    tiny = 2.0 ** -25 * (dtype is torch.float16)
    for name, a, da, b in (("grad_x", g, dg, w), ("grad_head", g.t().contiguous(), dg.t().contiguous(), x)):
        value, size = a @ b, a.abs() @ b.abs()
        room = da @ b.abs() + (b.shape[0] + 16) * F32 * size
        out[name] = (value, room + HALF[dtype] * (value.abs() + room) + tiny)
    return out


def close(got, want, name):
    value, room = want
    over = ((got.double() - value).abs() - room).max() if got.numel() else torch.zeros(())
    assert bool(((got.double() - value).abs() <= room).all()), (name, float(over))


def check(d, dtype, pad=0):
    rows, inner = d["x"].shape
    vocabulary = d["head"].shape[0]
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    gx = torch.full((rows + 1, inner + pad), 7.0, dtype=dtype, device="cuda")
    gh = torch.full((vocabulary + 1, inner + pad), 7.0, dtype=dtype, device="cuda")
    nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"], grad_x=gx[:rows, :inner], grad_head=gh[:vocabulary, :inner])
    want = definition(d, dtype)
    close(lse, want["lse"], "lse")
    close(loss, want["loss"], "loss")
    close(gx[:rows, :inner], want["grad_x"], "grad_x")
    close(gh[:vocabulary, :inner], want["grad_head"], "grad_head")
    for t, n in ((gx, rows), (gh, vocabulary)):
        assert bool((t[n:] == 7.0).all()) and bool((t[:, inner:] == 7.0).all())
    again = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    more = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])
    assert torch.equal(more[0], gx[:rows, :inner]) and torch.equal(more[1], gh[:vocabulary, :inner])


SIZES = [(1, 1, 1), (1, 2, 8), (2, 3, 3), (3, 7, 5), (5, 300, 64), (31, 129, 40), (33, 1000, 96), (64, 513, 24), (130, 1003, 97), (257, 515, 72),
         (300, 4100, 256), (2, 50_000, 128), (700, 33, 513), (1025, 130, 8), (2049, 264, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", SIZES)
def test_against_the_definition(sizes, dtype):
    seed = sum(sizes)
    check(problem(seed, *sizes, dtype, weighted=seed % 3 != 0, masked=0.3 if seed % 2 else 0.0), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(16, 1003, 512), (16, 517, 257), (15, 4100, 130), (9, 70, 1024), (1, 33, 2048), (16, 2000, 999), (4, 15, 4096), (16, 40_001, 24)])
def test_few_rows(sizes, dtype):
    check(problem(5, *sizes, dtype), dtype)
    check(problem(6, *sizes, dtype, pad=3), dtype, pad=3)
    d = problem(7, *sizes, dtype, masked=0.5)
    d["x"][d["label"] < 0] = float("nan")
    check(d, dtype)


@pytest.mark.parametrize("sizes", [(17, 1567, 2275), (64, 8192, 12), (64, 8193, 12), (63, 8129, 70), (100, 70, 4096), (33, 31, 5), (500, 1000, 65), (600, 1100, 130)])
def test_few_tiles_of_floats(sizes):
    for masked in (0.0, 0.4):
        check(problem(3, *sizes, torch.float32, masked=masked), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(2048, 8192, 64), (2100, 8200, 72), (4096, 2056, 320), (520, 16_384, 520)])
def test_large_tiles(sizes, dtype):
    check(problem(1, *sizes, dtype, masked=0.1), dtype)


@pytest.mark.parametrize("dtype,rows", [(torch.float32, 8200), (torch.bfloat16, 8200), (torch.float16, 9001)])
def test_pieces_of_the_vocabulary(dtype, rows):
    """More rows than g of a whole vocabulary has room for."""
    check(problem(2, rows, 20_003, 40, dtype, masked=0.2), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(511, 1000, 41), (512, 1000, 41), (600, 4097, 333), (2300, 9000, 131), (8300, 20_003, 41), (530, 40_000, 4097)])
def test_many_rows_that_start_anywhere(sizes, dtype):
    """Rows of odd lengths, copied or not, in one piece of the vocabulary or in several."""
    check(problem(12, *sizes, dtype, masked=0.2), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_many_rows_apart(dtype):
    check(problem(13, 700, 900, 56, dtype, masked=0.2, pad=3), dtype, 3)
    check(problem(13, 700, 900, 56, dtype, masked=0.2), dtype, 5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [1, 4, 8])
def test_rows_apart(dtype, pad):
    check(problem(3, 70, 333, 56, dtype, masked=0.2, pad=pad), dtype, pad)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("label", [torch.int32, torch.int64])
def test_rows_that_do_not_count(dtype, label):
    """Labels outside the vocabulary and weights of 0: zeros, whatever the rows hold, and the others as without them."""
    d = problem(4, 1100, 200, 48, dtype, label=label)
    out = torch.zeros(1100, dtype=torch.bool, device="cuda")
    for i, l in ((0, -1), (7, 200), (64, -100), (500, 2 ** 31 - 1), (1023, -2 ** 31), (1024, 201), (1099, -5)):
        d["label"][i] = l
        out[i] = True
    if label is torch.int64:
        d["label"][8], out[8] = 2 ** 40 + 3, True
    d["weight"][[1, 65, 1050]], out[[1, 65, 1050]] = 0.0, True
    d["x"][out] = float("nan")
    check(d, dtype)
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])
    assert bool((loss[out] == 0).all()) and bool((lse[out] == 0).all()) and bool((gx[out] == 0).all())
    keep = ~out
    few = nb.nacho_xent(d["x"][keep], d["head"], d["label"][keep], weight=d["weight"][keep])
    assert torch.equal(few[0], loss[keep]) and torch.equal(few[1], lse[keep])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,live", [((300, 5000, 300), (1, 40, 255, 256, 299)), ((1100, 3000, 520), (1, 130, 256, 257, 600)), ((70, 9000, 33), (1, 17, 33)),
                                        ((4200, 40_003, 264), (3, 2500))])
def test_few_of_many_rows_count(sizes, live, dtype):
    for n in live:
        d = problem(n, *sizes, dtype)
        order = torch.randperm(sizes[0], generator=torch.Generator().manual_seed(n)).cuda()
        d["label"][order[n:]] = -1
        check(d, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [32_767, 32_768, 33_793, 1_050_001])
def test_lists_of_many_rows(rows, dtype):
    """Rows that are counted before they are listed, a workgroup 1024 of them or more."""
    d = problem(rows, rows, 5, 8, dtype, masked=0.4, weighted=rows % 2 == 1, label=torch.int32 if rows % 2 else torch.int64)
    d["label"][2048:9000] = -1
    d["x"][d["label"] < 0] = float("nan")
    if rows % 2:
        d["weight"][20_000:20_050] = 0.0
        d["weight"][rows - 1] = 3.0                              # (the largest one, in the last workgroup)
        d["label"][rows - 1] = 2
    d["x"][rows - 1] = 1.0
    for last in (False, True):
        if last:
            d["label"].fill_(-1)
            d["label"][rows - 1] = 3
        loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
        gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])
        want = definition(d, dtype)
        # (The sum of a million rows' gradients passes the range of f16, whose numbers from 65520 on, the largest one and half a step, are
        # infinite: the value 67896.7 of 0.6 million rows is, and so may be any that its room brings there.)
        value, room = want["grad_head"]
        far = gh.isinf() & (value.abs() + room >= 65520) & (gh.sign() == value.sign()) if dtype is torch.float16 else torch.zeros_like(gh, dtype=torch.bool)
        close(lse, want["lse"], "lse")
        close(loss, want["loss"], "loss")
        close(gx, want["grad_x"], "grad_x")
        close(torch.where(far, value, gh.double()), want["grad_head"], "grad_head")
        again = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
        assert torch.equal(again[0], loss) and torch.equal(again[1], lse)


def test_the_time_of_listing_grows_as_the_rows():
    """Four times as many rows take about four times as long, not sixteen times."""
    times = []
    for rows in (1 << 22, 1 << 24):
        x, head = torch.ones((rows, 8), dtype=torch.bfloat16, device="cuda"), torch.ones((8, 8), dtype=torch.bfloat16, device="cuda")
        label = torch.zeros(rows, dtype=torch.int64, device="cuda")
        best = float("inf")
        for _ in range(4):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            nb.nacho_xent(x, head, label)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        times.append(best)
    assert times[1] <= 8 * times[0], times


@pytest.mark.parametrize("dtype", TYPES)
def test_no_row_counts(dtype):
    d = problem(5, 40, 300, 64, dtype)
    d["label"].fill_(-100)
    d["x"].fill_(float("nan"))
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"])
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse)
    for t in (loss, lse, gx, gh):
        assert bool((t == 0).all())
    for inner in (64, 63):
        x, head, label = d["x"][:0, :inner].contiguous(), d["head"][:, :inner].contiguous(), d["label"][:0]
        loss, lse = nb.nacho_xent(x, head, label)
        gx, gh = nb.nacho_xent_grad(x, head, label, lse)
        assert loss.shape == (0,) and gx.shape == (0, inner) and bool((gh == 0).all())


@pytest.mark.parametrize("rows", [5, 70])
def test_more_than_2_31_weights(rows):
    """Weights of the vocabulary's last words lie more than 2^32 bytes behind the first ones'; those between are zero."""
    vocabulary, inner = 140_000, 16_384
    g = torch.Generator(device="cuda").manual_seed(1)
    some = torch.tensor([0, 1, 77_777, 131_071, 131_072, 139_998, 139_999], device="cuda")
    head = torch.zeros((vocabulary, inner), dtype=torch.bfloat16, device="cuda")
    head[some] = (torch.randn((len(some), inner), generator=g, device="cuda") * 3 * inner ** -0.5).to(torch.bfloat16)
    x = torch.randn((rows, inner), generator=g, device="cuda").to(torch.bfloat16)
    label = some[torch.arange(rows, device="cuda") % len(some)]
    loss, lse = nb.nacho_xent(x, head, label)
    gx, gh = nb.nacho_xent_grad(x, head, label, lse)
    z, dz = x.double() @ head[some].double().T.contiguous(), (inner + 8) * F32 * (x.double().abs() @ head[some].double().abs().T.contiguous())
    all_z = torch.cat([z, torch.zeros((rows, 1), dtype=torch.float64, device="cuda").expand(-1, vocabulary - len(some))], dim=1)
    want = torch.logsumexp(all_z, dim=1)
    d_lse = dz.max(dim=1)[0] + 2.0 ** -21 + (64 + vocabulary / 2048) * F32 + 2 * F32 * want.abs()
    assert bool(((lse.double() - want).abs() <= d_lse).all())
    q = torch.exp(z - want[:, None]) - (label[:, None] == some).double()
    d_q = dz + d_lse[:, None] + 2.0 ** -18 + 2.0 ** -8 * q.abs()
    for got, value, room in ((gx, q @ head[some].double(), d_q @ head[some].double().abs()), (gh[some], q.T @ x.double(), d_q.T @ x.double().abs())):
        assert bool(((got.double() - value).abs() <= room * 1.01 + 2.0 ** -8 * value.abs() + 1e-6).all())


def test_weights_of_many_sizes():
    """f16 gradients under weights of one by a large number of rows, and under large ones: the probabilities do not vanish."""
    for size in (2.0 ** -14, 1.0, 2.0 ** 9):
        d = problem(6, 96, 2000, 64, torch.float16)
        d["weight"] *= size
        # (grad_head's values are f16 themselves: as many large ones as make them normal numbers)
        d["head"] = d["head"] / max(1.0, size ** 0.5)
        check(d, torch.float16)


def test_not_a_number_and_infinities():
    d = problem(7, 50, 300, 32, torch.float32)
    clean = nb.nacho_xent(d["x"], d["head"], d["label"])
    d["x"][3, 5], d["x"][9, 0] = float("nan"), float("inf")
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"])
    bad = torch.zeros(50, dtype=torch.bool, device="cuda")
    bad[[3, 9]] = True
    assert bool(loss[bad].isnan().all()) and bool(lse[bad].isnan().all())
    assert torch.equal(loss[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse)
    assert bool(gx[bad].isnan().all()) and not bool(gx[~bad].isnan().any()) and bool(gh.isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [5, 16, 50, 300])
@pytest.mark.parametrize("inner", [32, 33])
def test_infinite_weights(inner, rows, dtype):
    """A word whose logits are -inf has probability 0: the others are as without it.  Logits of +inf, or of -inf alone, leave no distribution."""
    word, column, vocabulary = 7, 4, 200
    d = problem(14, rows, vocabulary, inner, dtype)
    d["x"] = d["x"].abs() + 0.125
    d["label"][d["label"] == word] = 8
    others = torch.arange(vocabulary, device="cuda") != word
    without = {**d, "head": d["head"][others], "label": d["label"] - (d["label"] > word).long()}
    want = definition(without, dtype)
    d["head"][word, column] = -float("inf")
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])
    close(loss, want["loss"], "loss")
    close(lse, want["lse"], "lse")
    close(gh[others], want["grad_head"], "grad_head")
    assert bool((gh[word] == 0).all()) and bool(gx[:, column].isnan().all())
    rest = torch.arange(inner, device="cuda") != column
    close(gx[:, rest], tuple(t[:, rest] for t in want["grad_x"]), "grad_x")
    d["label"][0] = word
    again = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    assert float(again[0][0]) == float("inf") and torch.equal(again[0][1:], loss[1:]) and torch.equal(again[1], lse)
    for value, where in ((float("inf"), word), (float("nan"), word), (-float("inf"), slice(None))):
        head = d["head"].clone()
        head[where, column] = value
        loss, lse = nb.nacho_xent(d["x"], head, d["label"], weight=d["weight"])
        assert bool(loss.isnan().all()) and bool(lse.isnan().all())
        gx, gh = nb.nacho_xent_grad(d["x"], head, d["label"], lse, weight=d["weight"])
        assert bool(gx.isnan().all()) and bool(gh.isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [9, 16, 40])
def test_values_of_one_row_stay_its_own(rows, dtype):
    """A NaN, or infinities on both sides, in a row of x reach no other row's results; and all of grad_head."""
    d = problem(15, rows, 300, 64, dtype)
    clean = nb.nacho_xent(d["x"], d["head"], d["label"])
    first = nb.nacho_xent_grad(d["x"], d["head"], d["label"], clean[1], grad_head=False)[0]
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[3, rows - 1]] = True
    d["x"][3, 5], d["x"][rows - 1, 0] = float("nan"), float("inf")
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"])
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse)
    assert bool(loss[bad].isnan().all()) and bool(lse[bad].isnan().all()) and bool(gx[bad].isnan().all()) and bool(gh.isnan().all())
    assert torch.equal(loss[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad]) and torch.equal(gx[~bad], first[~bad])


def test_logits_far_apart():
    """Logits of thousands: the softmax is one column."""
    d = problem(8, 20, 130, 16, torch.float32, size=2000.0)
    check(d, torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_that_are_not_wanted(dtype):
    d = problem(9, 300, 700, 40, dtype, masked=0.2)
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"])
    both = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse)
    one, none = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, grad_head=False)
    assert none is None and torch.equal(one, both[0])
    none, one = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, grad_x=False)
    assert none is None and torch.equal(one, both[1])


def test_gradients_against_differences():
    """Central differences of the loss along random directions, in 32 bits.  With M the largest change of a row's logits along the
    direction, the third derivative of its lse is at most 8 M^3; the losses themselves are off by `room`."""
    d = problem(10, 40, 200, 48, torch.float32)
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])
    room = float(definition(d, torch.float32)["loss"][1].sum())
    step = 2.0 ** -5
    for name, grad in (("x", gx), ("head", gh)):
        torch.manual_seed(1)
        u = torch.randn_like(d[name]) / 8
        change = u @ d["head"].T if name == "x" else d["x"] @ u.T
        ends = []
        for sign in (1, -1):
            moved = {**d, name: d[name] + sign * step * u}
            ends.append(nb.nacho_xent(moved["x"], moved["head"], d["label"], weight=d["weight"])[0].double().sum())
        slope = float(ends[0] - ends[1]) / (2 * step)
        third = 8 * float((d["weight"].double() * change.double().abs().max(dim=1)[0] ** 3).sum())
        assert abs(slope - float((grad.double() * u.double()).sum())) <= third * step ** 2 / 6 + 2 * room / step


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(1, 1, 1), (16, 32_768, 1025), (16, 32_769, 1025), (16, 24_575, 64), (17, 16_384, 40), (64, 8192, 12), (64, 8193, 12), (100, 5000, 7),
                                   (600, 4097, 333), (2100, 8200, 72), (8200, 20_003, 40), (33_000, 70, 16)])
def test_workspaces_are_enough(sizes, dtype):
    """Calls with workspaces of the bytes that were asked for write nothing behind them, and give what those with their own give."""
    d = problem(16, *sizes, dtype, masked=0.1)
    c = nb._xent_layer(d["x"], d["head"], d["label"], d["weight"])
    rooms = []
    for name in ("nacho_xent_workspace_bytes", "nacho_xent_grad_workspace_bytes"):
        need = nb.C.c_size_t(0)
        assert getattr(nb.lib(), name)(nb.C.byref(c), nb.C.byref(need)) == 0
        rooms.append(torch.full((need.value + (1 << 20),), 0x5a, dtype=torch.uint8, device="cuda"))
    first, second = (room[:-(1 << 20)] for room in rooms)
    loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"], ws=first)
    gx, gh = nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"], ws=second)
    assert all(bool((room[-(1 << 20):] == 0x5a).all()) for room in rooms)
    own = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
    own += nb.nacho_xent_grad(d["x"], d["head"], d["label"], own[1], weight=d["weight"])
    assert all(torch.equal(a, b) for a, b in zip((loss, lse, gx, gh), own))
    want = definition(d, dtype)
    close(loss, want["loss"], "loss")
    close(lse, want["lse"], "lse")


def test_lists_of_many_rows_under_a_captured_graph():
    d = problem(17, 40_000, 20, 16, torch.float16, masked=0.2)

    def work():
        loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
        return [loss, lse, *nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])]

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = work()
    for seed in range(4):
        torch.manual_seed(seed)
        d["x"].normal_()
        d["label"].random_(-10, 25)
        d["weight"].uniform_(0.0, 1.0 + seed)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(result, work()))
        torch.cuda.synchronize()


def test_on_another_stream_and_under_captured_graphs():
    d = problem(11, 400, 3000, 64, torch.bfloat16, masked=0.2)

    def work():
        loss, lse = nb.nacho_xent(d["x"], d["head"], d["label"], weight=d["weight"])
        return [loss, lse, *nb.nacho_xent_grad(d["x"], d["head"], d["label"], lse, weight=d["weight"])]

    want = work()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = work()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, results = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            results.append(work())
    for seed in range(4):
        torch.manual_seed(seed)
        d["x"].normal_()
        d["label"].random_(-500, 3000)
        graphs[0].replay()
        torch.cuda.synchronize()
        eager = work()
        graphs[1].replay()
        torch.cuda.synchronize()
        for result in results:
            assert all(torch.equal(a, b) for a, b in zip(result, eager))
