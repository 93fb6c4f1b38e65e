"""What the Python side of the training operators makes and refuses before the library is called (the library's calls are
replaced, nothing is launched, no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_17198_amd import binding as nb


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's calls, none of which is made; host tensors stand for those of a GPU."""
    made = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                made.append(name)
                if name.endswith("_workspace_bytes"):
                    C.cast(args[-1], C.POINTER(C.c_size_t))[0] = 256
                return 0
            return call

    monkeypatch.setattr(nb, "lib", lambda: Library())
    monkeypatch.setattr(nb, "_stream", lambda: 0)
    monkeypatch.setattr(nb, "_HOST", None)
    monkeypatch.setattr(nb, "_current_device", lambda: -1)
    return made


def ints(*values):
    return torch.tensor(values, dtype=torch.int32)


def teacher(rows=3, cols=20):
    return nb.csr(torch.arange(rows + 1, dtype=torch.int32) * 2, ints(*[1, 5] * rows), rows, cols, torch.zeros(2 * rows, dtype=torch.float32))


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_results_do_not_take_the_default_type(calls, default):
    """A program that sets torch's default type gets results of the types that the library writes."""
    before = torch.get_default_dtype()
    try:
        torch.set_default_dtype(default)
        z = torch.zeros((3, 20), dtype=torch.bfloat16)
        loss, lse = nb.nacho_distill(teacher(), z)
        r = nb.nacho_route(z, 2)
        y = torch.zeros((6, 20), dtype=torch.float16)
        _, grad_gate = nb.nacho_combine_grad(ints(0, 2, 4, 6), ints(0, 1, 2, 3, 4, 5), y, y[:3])
        for t in (loss, lse, r.gate, r.lse, r.balance, grad_gate):
            assert t.dtype is torch.float32
        for t in (nb.nacho_distill_grad(teacher(), z, lse), nb.nacho_route_grad(z, r)):
            assert t.dtype is z.dtype
    finally:
        torch.set_default_dtype(before)


def test_weights_whose_rows_lie_on_each_other_are_refused(calls):
    """Expanded weights (distance 0 between rows) are not what a leading dimension of their length reads, past their end."""
    x, bounds, token = torch.zeros((5, 16)), ints(0, 3, 7), ints(0, 1, 2, 3, 4, 0, 1)
    row, flat, y = torch.zeros((2, 1, 16)), torch.zeros((1, 24, 16)), torch.zeros((7, 24))
    whole = torch.zeros((2, 24, 16))
    for weight in (row.expand(2, 24, 16), row[:1].expand(2, 24, 16), torch.zeros(16).expand(2, 24, 16)):
        with pytest.raises(ValueError):
            nb.nacho_experts(x, weight, bounds, token=token)
        with pytest.raises(ValueError):
            nb.nacho_experts_grad(y, x, weight, bounds, token=token)
        with pytest.raises(ValueError):
            nb.nacho_experts_grad(y, x, whole, bounds, token=token, grad_weight=weight)
    assert "nacho_experts" not in calls and "nacho_experts_grad" not in calls
    # (one row or one expert may have any distance; padded rows and experts have their own)
    assert nb._stack(row.expand(2, 1, 16), "w", (2, 1, 16), torch.float32, row.device) == (16, 16)
    assert nb._stack(flat, "w", (1, 24, 16), torch.float32, flat.device) == (16, 24 * 16)
    assert nb._stack(torch.zeros((2, 30, 20))[:, :24, :16], "w", (2, 24, 16), torch.float32, flat.device) == (20, 600)


def test_host_tensors_are_refused():
    z, x, w, y = torch.zeros((3, 20)), torch.zeros((5, 16)), torch.zeros((2, 20, 16)), torch.zeros((6, 20))
    bounds, token, pos, slot = ints(0, 3, 6), ints(0, 1, 2, 3, 4, 0), ints(0, 2, 4, 6), ints(0, 1, 2, 3, 4, 5)
    floats, r = torch.zeros(3), nb.Routing(3, 20, 2, z.device)
    for call in (lambda: nb.nacho_distill(teacher(), z), lambda: nb.nacho_distill(teacher(), z, grad=torch.zeros_like(z)),
                 lambda: nb.nacho_distill_grad(teacher(), z, floats), lambda: nb.nacho_route(z, 2), lambda: nb.nacho_route(z, 2, out=r),
                 lambda: nb.nacho_route_grad(z, r), lambda: nb.nacho_experts(x, w, bounds, token=token),
                 lambda: nb.nacho_experts_grad(y, x, w, bounds, token=token), lambda: nb.nacho_combine(pos, slot, y),
                 lambda: nb.nacho_combine_grad(pos, slot, y, z)):
        with pytest.raises(ValueError):
            call()


def test_workspaces_and_routings_elsewhere_are_refused(calls):
    """(the device `meta` stands for another one than that of the rows)"""
    z, other = torch.zeros((3, 20)), torch.empty(1 << 20, dtype=torch.uint8, device="meta")
    x, w, bounds = torch.zeros((6, 16)), torch.zeros((2, 20, 16)), ints(0, 3, 6)
    strange = nb.Routing(3, 20, 2, z.device)
    strange.pos = strange.pos.to("meta")
    for call in (lambda: nb.nacho_distill(teacher(), z, ws=other), lambda: nb.nacho_route(z, 2, ws=other),
                 lambda: nb.nacho_route(z, 2, ws=torch.zeros(1 << 20, dtype=torch.uint8)[::2]), lambda: nb.nacho_route_grad(z, strange),
                 lambda: nb.nacho_experts_grad(torch.zeros((6, 20)), x, w, bounds, ws=other)):
        with pytest.raises(ValueError):
            call()
    assert not [c for c in calls if not c.endswith("_bytes")]


def test_operands_arrays_lie_together():
    """Arrays of one operand that have gaps, or that lie on several devices, make no descriptor."""
    pos, crd, val = ints(0, 2, 4), ints(1, 5, 2, 3), torch.zeros(4)
    gaps = lambda t: torch.stack([t, t], dim=1)[:, 0]
    for p, c, v in ((gaps(pos), crd, val), (pos, gaps(crd), val), (pos, crd, gaps(val)), (pos.to("meta"), crd, val), (pos, crd.to("meta"), val),
                    (pos, crd, val.to("meta"))):
        with pytest.raises(ValueError):
            nb.csr(p, c, 2, 9, v)
    assert nb.csr(pos, crd, 2, 9, val).nnz == 4
    rows = ints(0, 1, 1, 2)
    with pytest.raises(ValueError):
        nb.coo(gaps(rows), crd, 3, 9, val)


def test_gradients_that_are_not_wanted(monkeypatch, calls):
    """False for a gradient: no array is made, NULL goes to the library, None comes back."""
    given = {}

    class Library:
        def __getattr__(self, name):
            def call(*args):
                given[name] = args
                if name.endswith("_workspace_bytes"):
                    C.cast(args[-1], C.POINTER(C.c_size_t))[0] = 256
                return 0
            return call

    monkeypatch.setattr(nb, "lib", lambda: Library())
    x, w, y, bounds = torch.zeros((6, 16)), torch.zeros((2, 20, 16)), torch.zeros((6, 20)), ints(0, 3, 6)
    for gx, gw in ((None, False), (False, None), (False, False)):
        a, b = nb.nacho_experts_grad(y, x, w, bounds, grad_x=gx, grad_weight=gw, grad_bias=torch.zeros((2, 20)))
        args = given["nacho_experts_grad"]
        assert (a is None) == (gx is False) == (args[5] is None) and (b is None) == (gw is False) == (args[7] is None) and args[10] is not None
    pos, slot, go = ints(0, 2, 4, 6), ints(0, 1, 2, 3, 4, 5), torch.zeros((3, 20))
    for gy, gg in ((None, False), (False, None), (False, False)):
        a, b = nb.nacho_combine_grad(pos, slot, y, go, grad_y=gy, grad_gate=gg)
        args = given["nacho_combine_grad"]
        assert (a is None) == (gy is False) == (args[7] is None) and (b is None) == (gg is False) == (args[9] is None)
