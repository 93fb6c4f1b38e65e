"""nacho_experts, nacho_experts_grad against the definition in 64 bits.

Tolerances: a sum of n products held in 32 bits is within (n + 8) 2^-24 of the sum of their magnitudes; activations add a few
2^-24 of their argument; results of 16 bits are rounded once (2^-8 of a bf16, 2^-11 of an f16, half the smallest f16
step).  On the way back the gradient before the activation is rounded to the type as well, and taken from rows before
the activation that were: every term of a product is off by twice that rounding of the term (the slopes of gelu and silu
change by less than their argument does, next to a value of one)."""
import math

import numpy as np
import pytest
import torch

from paper_2604_17198_amd import binding as nb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
STEP = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ACTS = ["none", "relu", "gelu", "silu"]


def act64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        q = torch.sigmoid(z)
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def problem(seed, counts, tokens, inner, outer, dtype, bias, gather=True, pad=0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g)
    experts, slots = len(counts), sum(counts)
    bounds = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)
    token = torch.randint(0, tokens, (slots,), generator=g, dtype=torch.int32) if gather else None
    rows = tokens if gather else slots
    d = dict(x=rand(rows, inner + pad).to(dtype)[:, :inner], w=(rand(experts, outer, inner + pad) / math.sqrt(inner)).to(dtype)[:, :, :inner],
             bias=rand(experts, outer).to(dtype) if bias else None, gy=rand(slots, outer + pad).to(dtype)[:, :outer], bounds=bounds, token=token)
    return d


def to_gpu(d):
    """Copies that keep the strides."""
    def move(t):
        if t is None:
            return None
        base = t._base if t._base is not None else t
        return base.cuda().as_strided(t.shape, t.stride(), t.storage_offset())
    return {k: move(v) for k, v in d.items()}


def close(got, want, size, terms, step, dtype, what):
    g = got.cpu().double()
    room = step * want.abs() + (terms + 8) * 2.0 ** -24 * size + 2.0 ** -25 * (dtype is torch.float16)
    assert bool(((g - want).abs() <= room).all()), (what, ((g - want).abs() - room).max())


def check(d, act, dtype, forward_only=False, pad=0):
    bounds, slots = d["bounds"].tolist(), d["bounds"][-1].item()
    experts, outer, inner = d["w"].shape
    x, w, gy = d["x"].double(), d["w"].double(), d["gy"].double()
    xs = x[d["token"].long()] if d["token"] is not None else x
    g = to_gpu(d)
    room = slots + 3                                         # places behind the last slot
    y = torch.full((room, outer + pad), 7.0, dtype=dtype, device="cuda")
    pre = torch.full((room, outer + pad), 7.0, dtype=dtype, device="cuda")
    token = g["token"]
    if token is not None:
        token = torch.cat([token, torch.full((3,), -1, dtype=torch.int32, device="cuda")])
        xg = g["x"]
    else:
        xg = torch.cat([g["x"], torch.full((3, inner), float("nan"), dtype=dtype, device="cuda")])
    nb.nacho_experts(xg, g["w"], g["bounds"], token=token, bias=g["bias"], act=act, y=y[:, :outer], pre=pre[:, :outer])
    step, eps = STEP[dtype], 0.0 if dtype is torch.float32 else STEP[dtype]
    zs = []
    for e in range(experts):
        a, b = bounds[e], bounds[e + 1]
        z = xs[a:b] @ w[e].T
        size = xs[a:b].abs() @ w[e].abs().T
        if d["bias"] is not None:
            z, size = z + d["bias"][e].double(), size + d["bias"][e].double().abs()
        zs.append(z)
        close(pre[a:b, :outer], z, size, inner, step, dtype, ("pre", e))
        close(y[a:b, :outer], act64(z, act), 1.2 * size + z.abs() * 4, inner, step, dtype, ("y", e))
    assert bool((y[slots:] == 7.0).all()) and bool((y[:, outer:] == 7.0).all()) and bool((pre[:, outer:] == 7.0).all())
    plain = nb.nacho_experts(xg, g["w"], g["bounds"], token=token, bias=g["bias"], act=act)
    assert torch.equal(plain[:slots], y[:slots, :outer])
    if forward_only:
        return
    gyg = torch.cat([g["gy"], torch.full((3, outer), float("nan"), dtype=dtype, device="cuda")])
    gx = torch.full((room, inner + pad), 7.0, dtype=dtype, device="cuda")
    gw = torch.full((experts, outer, inner + pad), 7.0, dtype=dtype, device="cuda")
    gb = torch.full((experts, outer), 7.0, dtype=dtype, device="cuda")
    nb.nacho_experts_grad(gyg, xg, g["w"], g["bounds"], token=token, act=act, pre=pre[:, :outer] if act != "none" else None,
                          grad_x=gx[:, :inner], grad_weight=gw[:, :, :inner], grad_bias=gb)
    kept = pre[:slots, :outer].cpu().double()
    for e in range(experts):
        a, b = bounds[e], bounds[e + 1]
        # (from the rows that were kept, which relu's edge needs, and rounded to the type as the definition has it)
        gz = (gy[a:b] * slope64(kept[a:b], act)).to(dtype).double()
        room_gz = gy[a:b].abs() * (slope64(kept[a:b], act).abs() + 2.0 ** -20)
        close(gx[a:b, :inner], gz @ w[e], room_gz @ w[e].abs(), outer + 2 * eps * 2.0 ** 24, step, dtype, ("grad_x", e))
        close(gw[e][:, :inner], gz.T @ xs[a:b], room_gz.T @ xs[a:b].abs(), (b - a) + 2 * eps * 2.0 ** 24, step, dtype, ("grad_w", e))
        close(gb[e], gz.sum(0), room_gz.sum(0), (b - a) + 2 * eps * 2.0 ** 24, step, dtype, ("grad_bias", e))
    assert bool((gx[slots:] == 7.0).all()) and bool((gx[:, inner:] == 7.0).all()) and bool((gw[:, :, inner:] == 7.0).all())


CASES = [([1], 1, 1, 1), ([3], 5, 8, 8), ([0, 2, 0], 4, 16, 24), ([5, 1, 130], 40, 32, 64), ([17, 16, 15], 9, 40, 136),
         ([128, 129, 127], 200, 64, 128), ([300, 0, 7, 64], 100, 200, 264), ([33, 260], 64, 512, 96), ([2, 3, 1, 0, 4], 3, 1024, 256),
         ([9, 70], 30, 33, 65), ([140, 5], 80, 127, 131), ([1, 1, 1], 2, 257, 3), ([600], 300, 96, 72), ([20, 40], 16, 8, 1000)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts,tokens,inner,outer", CASES)
def test_layer_and_gradients(counts, tokens, inner, outer, dtype):
    at = CASES.index((counts, tokens, inner, outer))
    check(problem(at, counts, tokens, inner, outer, dtype, at % 2 == 0), ACTS[at % 4], dtype)


ODD = [([300, 0, 90], 200, 5, 7), ([40, 3], 30, 3, 300), ([70, 129], 90, 301, 6), ([700, 260, 1], 400, 131, 261),
       ([2100, 1500, 0, 900], 1000, 67, 2051), ([33, 64, 65, 31, 32], 50, 129, 515)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts,tokens,inner,outer", ODD)
def test_rows_that_no_word_fits(counts, tokens, inner, outer, dtype):
    """Rows shorter than 16 bytes, and longer ones of odd lengths: one step of the sum, a few and many, ended early or not."""
    at = ODD.index((counts, tokens, inner, outer))
    check(problem(40 + at, counts, tokens, inner, outer, dtype, at % 2 == 0), ACTS[at % 4], dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("pad", [0, 8, 5])
def test_activations_strides_and_rows_in_place(act, pad, dtype):
    check(problem(5, [40, 0, 150, 3], 60, 72, 104, dtype, True, gather=False, pad=pad), act, dtype, pad=pad)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_many_experts(dtype):
    rng = np.random.default_rng(1)
    counts = rng.integers(0, 4, 150).tolist()
    check(problem(6, counts, 50, 48, 40, dtype, True), "silu", dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_no_slots(dtype):
    d = problem(7, [0, 0], 4, 16, 24, dtype, True)
    check(d, "gelu", dtype)
    y = nb.nacho_experts(torch.empty((0, 16), dtype=dtype, device="cuda"), d["w"].cuda(), d["bounds"].cuda())
    assert y.shape == (0, 24)
    gx, gw = nb.nacho_experts_grad(y, torch.empty((0, 16), dtype=dtype, device="cuda"), d["w"].cuda(), d["bounds"].cuda())
    assert gx.shape == (0, 16) and not bool(gw.any())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inner", [64, 61])
def test_one_experts_values_stay_its_own(inner, dtype):
    """Infinities and NaN in one expert's weights, and in rows of x that its slots alone read, reach no other's results."""
    d = problem(8, [37, 50, 41], 128, inner, 40, dtype, False)
    token = torch.cat([torch.arange(37), 37 + torch.arange(50), 87 + torch.arange(41)]).to(torch.int32)
    x, w, gy = (d[k].clone() for k in ("x", "w", "gy"))
    x[37:87], w[1], gy[37:87] = float("inf"), float("nan"), float("nan")
    run = lambda x, w, gy: (nb.nacho_experts(x.cuda(), w.cuda(), d["bounds"].cuda(), token=token.cuda()),
                            *nb.nacho_experts_grad(gy.cuda(), x.cuda(), w.cuda(), d["bounds"].cuda(), token=token.cuda()))
    for spoilt, clean, by in zip(run(x, w, gy), run(d["x"], d["w"], d["gy"]), ("slot", "slot", "expert")):
        keep = [0, 2] if by == "expert" else list(range(37)) + list(range(87, 128))
        assert torch.equal(spoilt[keep], clean[keep])
        assert bool(torch.isnan(spoilt[1 if by == "expert" else slice(37, 87)]).all())


def test_gradient_against_differences():
    """Central differences of sum(y h) in 64 bits; error step^2 / 6 times a third derivative below 10."""
    d = problem(9, [3, 4], 5, 6, 7, torch.float32, True)
    bounds, token, h = d["bounds"].tolist(), d["token"].long(), d["gy"].double()

    def objective(x, w, b):
        return sum((act64(x[token[bounds[e]:bounds[e + 1]]] @ w[e].T + b[e], "gelu") * h[bounds[e]:bounds[e + 1]]).sum() for e in range(2)).item()

    g = to_gpu(d)
    pre, gb = torch.empty((7, 7), device="cuda"), torch.empty((2, 7), device="cuda")
    nb.nacho_experts(g["x"], g["w"], g["bounds"], token=g["token"], bias=g["bias"], act="gelu", pre=pre)
    gx, gw = nb.nacho_experts_grad(g["gy"], g["x"], g["w"], g["bounds"], token=g["token"], act="gelu", pre=pre, grad_bias=gb)
    by_token = torch.zeros((5, 6), dtype=torch.float64).index_add_(0, token, gx.cpu().double())
    at = [d["x"].double(), d["w"].double(), d["bias"].double()]
    for which, grad in enumerate((by_token, gw.cpu().double(), gb.cpu().double())):
        for i in range(grad.numel()):
            ends = []
            for sign in (1e-4, -1e-4):
                moved = [t.clone() for t in at]
                moved[which].view(-1)[i] += sign
                ends.append(objective(*moved))
            assert abs((ends[0] - ends[1]) / 2e-4 - grad.reshape(-1)[i].item()) <= 3e-5


def test_offsets_past_two_to_the_31():
    """A last expert whose weights lie past 2^31 elements, and rows of y past them."""
    experts, outer, inner = 70, 5600, 5600                   # 2.2e9 elements, 4.4 GB
    w = torch.zeros((experts, outer, inner), dtype=torch.bfloat16, device="cuda")
    w[-1].fill_(2.0 ** -4)
    bounds = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    bounds[-1] = 3
    x = torch.ones((3, inner), dtype=torch.bfloat16, device="cuda")
    y = nb.nacho_experts(x, w, bounds)
    assert bool((y == 350).all())
    gx, gw = nb.nacho_experts_grad(torch.ones_like(y), x, w, bounds)
    assert bool((gx == 350).all()) and bool((gw[-1] == 3).all()) and not bool(gw[0].any())


def test_another_stream_and_the_same_bits_again():
    d = to_gpu(problem(10, [100, 30, 200], 64, 160, 320, torch.bfloat16, True))

    def run():
        pre, gb = torch.empty((330, 320), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 320), dtype=torch.bfloat16, device="cuda")
        y = nb.nacho_experts(d["x"], d["w"], d["bounds"], token=d["token"], bias=d["bias"], act="silu", pre=pre)
        return [y, pre, gb, *nb.nacho_experts_grad(d["gy"], d["x"], d["w"], d["bounds"], token=d["token"], act="silu", pre=pre, grad_bias=gb)]

    first = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_refusals():
    d = to_gpu(problem(11, [3, 4], 5, 16, 24, torch.float32, True))
    call = lambda **more: nb.nacho_experts(**{**dict(x=d["x"], weight=d["w"], expert_pos=d["bounds"], token=d["token"]), **more})
    with pytest.raises(TypeError):
        call(x=d["x"].double(), weight=d["w"].double())
    for wrong in (dict(weight=d["w"].half()), dict(weight=d["w"][0]), dict(expert_pos=d["bounds"].long()), dict(expert_pos=d["bounds"][:2]),
                  dict(token=d["token"].long()), dict(act="tanh"), dict(bias=d["bias"][:, :3]), dict(y=torch.empty((7, 23), device="cuda")),
                  dict(x=d["x"].t().contiguous().t())):
        with pytest.raises(ValueError):
            call(**wrong)
    big = torch.empty((7, 24), device="cuda")
    with pytest.raises(nb.NachoError):
        call(y=big, pre=big)
    gy = torch.empty((7, 24), device="cuda")
    with pytest.raises(nb.NachoError):
        nb.nacho_experts_grad(gy, d["x"], d["w"], d["bounds"], token=d["token"], act="gelu")
    with pytest.raises(nb.NachoError):
        nb.nacho_experts_grad(gy, d["x"], d["w"], d["bounds"], token=d["token"], act="gelu", pre=torch.empty_like(gy),
                              ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(nb.NachoError):
        nb.nacho_experts_grad(gy, d["x"], d["w"], d["bounds"], token=d["token"], grad_weight=d["w"])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts,inner,outer", [([1500, 700], 72, 8200), ([530, 513], 200, 16384), ([600, 900, 4], 8200, 264)])
def test_the_largest_tiles(counts, inner, outer, dtype):
    """Enough slots an expert, and enough of them, for tiles of 256 x 256 in every direction, with rows and columns left over."""
    check(problem(20, counts, 300, inner, outer, dtype, True), "silu", dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inner", [64, 128, 192, 256, 264, 320, 136])
def test_steps_of_the_sum(inner, dtype):
    """Even and odd numbers of whole steps of k, and parts of one behind them, in all three products."""
    check(problem(21, [64 + inner, 130, inner // 2, 1], 90, inner, 384 - inner // 2, dtype, False), "none", dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("outer", [96, 101, 3])
def test_bias_gradients_are_rounded_once(outer, act, dtype):
    """Sums of what the rows' gradients are before they are rounded to the type: a rounding of the sum, n 2^-24 of the terms for a
    sum in 32 bits, and 2^-20 of a term's factor for slopes of 16-bit rows."""
    g = torch.Generator().manual_seed(outer)
    counts, inner = [900, 0, 70], 8
    bounds = torch.tensor([0, 900, 900, 970], dtype=torch.int32)
    pre, gy = ((torch.randn((970, outer), generator=g) * 1.5).to(dtype) for _ in range(2))
    x, w = torch.zeros((970, inner), dtype=dtype, device="cuda"), torch.zeros((3, outer, inner), dtype=dtype, device="cuda")
    gb = torch.full((3, outer), 7.0, dtype=dtype, device="cuda")
    nb.nacho_experts_grad(gy.cuda(), x, w, bounds.cuda(), act=act, pre=pre.cuda(), grad_bias=gb)
    for e in range(3):
        a, b = bounds[e], bounds[e + 1]
        term = gy[a:b].double() * slope64(pre[a:b].double(), act)
        size = (gy[a:b].double().abs() * (slope64(pre[a:b].double(), act).abs() * (counts[e] + 8) * 2.0 ** -24 + 2.0 ** -20)).sum(0)
        room = STEP[dtype] * term.sum(0).abs() + size + 2.0 ** -25 * (dtype is torch.float16)
        assert bool(((gb[e].cpu().double() - term.sum(0)).abs() <= room).all()), e


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act,outer", [("relu", 24), ("gelu", 24), ("silu", 24), ("gelu", 13), ("silu", 13)])
def test_slopes_of_rows_past_the_types_range(act, outer, dtype):
    """A row before the activation that left its type's range is kept as an infinity: slope 0 below and 1 above, as of any
    number as far out; a NaN stays one."""
    far = torch.tensor([float("-inf"), float("inf"), torch.finfo(dtype).min, torch.finfo(dtype).max], dtype=dtype)
    pre = far[:, None].expand(4, outer).contiguous()
    bounds = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    x, w = torch.ones((4, 8), dtype=dtype, device="cuda"), torch.ones((1, outer, 8), dtype=dtype, device="cuda")
    gb = torch.empty((1, outer), dtype=dtype, device="cuda")
    gx, gw = nb.nacho_experts_grad(torch.ones((4, outer), dtype=dtype, device="cuda"), x, w, bounds, act=act, pre=pre.cuda(), grad_bias=gb)
    assert gx[:, 0].tolist() == [0, outer, 0, outer] and bool((gb == 2).all()) and bool((gw == 2).all())
    pre[2, 1] = float("nan")
    gx, gw = nb.nacho_experts_grad(torch.ones((4, outer), dtype=dtype, device="cuda"), x, w, bounds, act=act, pre=pre.cuda(), grad_bias=gb)
    assert torch.isnan(gx[:, 0]).tolist() == [False, False, True, False] and bool(torch.isnan(gb[0, 1])) and bool((gb[0, 2:] == 2).all())


def test_slots_up_to_the_last_of_two_to_the_31():
    """An expert whose slots start at any place and end at the last that there can be: sums of places pass 31 bits."""
    slots = 2 ** 31 - 1                                      # rows of one element: 4.3 GB each
    bounds = torch.tensor([0, 5, slots], dtype=torch.int32, device="cuda")
    x = torch.full((slots, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    x[4], x[-1] = 3.0, 5.0
    w = torch.tensor([3.0, 7.0], dtype=torch.bfloat16, device="cuda").reshape(2, 1, 1)
    y = torch.zeros_like(x)
    nb.nacho_experts(x, w, bounds, y=y)
    assert y[:5, 0].tolist() == [6, 6, 6, 6, 9] and y[-1].item() == 35 and bool((y[5:-1] == 14).all())
    x[-2] = -1.0                                             # (as rows before the activation)
    y.fill_(1.0)
    gx, _ = nb.nacho_experts_grad(y, x, w, bounds, act="relu", pre=x, grad_weight=False)
    assert bool((gx[:5] == 3).all()) and gx[-2].item() == 0 and gx[-1].item() == 7 and bool((gx[5:-2] == 7).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts,inner,outer", [([520, 700], 16392, 264), ([577, 1100, 0], 16640, 264), ([520, 700], 16391, 263)])
def test_the_largest_tiles_on_the_way_back(counts, inner, outer, dtype):
    """512 slots an expert and more, and enough columns, for the largest tiles of each type in both gradients: whole steps of the
    sum, even and odd numbers of them, and what is left of one; rows and columns that end inside a tile; an expert without a slot."""
    check(problem(22, counts, 300, inner, outer, dtype, True), "gelu", dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_many_experts_of_some_hundred_slots(dtype):
    """Fewer slots an expert than the largest tiles are for, and enough of all for tiles of 128 x 128 in all three products."""
    counts = np.random.default_rng(23).integers(150, 450, 16).tolist()
    check(problem(23, counts, 700, 2064, 2056, dtype, True), "relu", dtype)
