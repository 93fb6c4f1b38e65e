"""What the training operators refuse, asked of the built library with made-up addresses (nothing is launched, no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_17198_amd import binding as nb

BAD, UNSUPPORTED, WORKSPACE, HIP = -1, -2, -3, -5
A, B, D, E = 1 << 40, 2 << 40, 3 << 40, 4 << 40              # addresses far apart


def teacher(rows=4, cols=100, stored=10, pos=A, crd=A + 4096, val=A + 8192, kinds=(nb.DENSE, nb.COMPRESSED), levels=2):
    t = nb._Tensor()
    t.nlevels = levels
    t.lvl[0].kind, t.lvl[0].extent = kinds[0], rows
    t.lvl[1].kind, t.lvl[1].extent, t.lvl[1].pos, t.lvl[1].crd, t.lvl[1].count = kinds[1], cols, pos, crd, stored
    t.val = val
    return t


def size(f, *a):
    n = C.c_size_t(0)
    rc = f(*a, C.byref(n))
    return rc, n.value


def test_distill():
    lib = nb.lib()

    def call(t=None, logits=B, ldl=100, dtype=nb.F32, tau=1.0, loss=E, lse=E + 4096, grad=None, ldg=0, ws=None, n=0):
        return lib.nacho_distill(C.byref(t or teacher()), logits, ldl, dtype, None, tau, loss, lse, grad, ldg, ws, n, None)

    assert call(logits=None) == BAD and call(ldl=99) == BAD and call(logits=B + 2) == BAD and call(dtype=nb.F64) == BAD
    assert call(loss=None) == BAD and call(lse=None) == BAD and lib.nacho_distill(None, B, 100, nb.F32, None, 1.0, E, E, None, 0, None, 0, None) == BAD
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-38):
        assert call(tau=tau) == BAD
    assert call(grad=D, ldg=99) == BAD and call(grad=B + 400, ldg=100) == BAD and call(grad=D + 1, ldg=100) == BAD
    assert call(teacher(kinds=(nb.COMPRESSED, nb.COMPRESSED))) == UNSUPPORTED and call(teacher(levels=1)) == UNSUPPORTED
    assert call(teacher(pos=None)) == BAD and call(teacher(crd=None)) == BAD and call(teacher(val=None)) == BAD and call(teacher(crd=A + 4)) == BAD
    # few long rows are cut into parts, which need room
    assert size(lib.nacho_distill_workspace_bytes, 2, 1 << 20, nb.F32)[1] > 0 and size(lib.nacho_distill_workspace_bytes, 4000, 1000, nb.F32) == (0, 0)
    assert call(teacher(rows=2, cols=1 << 20), ldl=1 << 20) == WORKSPACE
    assert size(lib.nacho_distill_workspace_bytes, -1, 5, nb.F32)[0] == BAD
    assert lib.nacho_distill_grad(C.byref(teacher()), B, 100, nb.BF16, None, 1.0, None, D, 100, None) == BAD
    assert lib.nacho_distill_grad(C.byref(teacher()), B, 100, nb.BF16, None, 1.0, E, None, 100, None) == BAD


def test_route():
    lib = nb.lib()
    full = nb._Routing(*[A + 4096 * i for i in range(10)])
    n = size(lib.nacho_route_workspace_bytes, 100, 16, 2)[1]

    def call(logits=B, ldl=16, tokens=100, experts=16, dtype=nb.F32, k=2, out=full, ws=D, room=n):
        return lib.nacho_route(logits, ldl, tokens, experts, dtype, k, 0, None, C.byref(out) if out else None, ws, room, None)

    assert n > 0 and call(logits=None) == BAD and call(ldl=15) == BAD and call(dtype=nb.F64) == BAD and call(out=None) == BAD
    assert call(k=0) == BAD and call(k=17) == BAD and call(tokens=-1) == BAD and call(experts=0) == BAD
    assert call(experts=1025, ldl=1025) == UNSUPPORTED and call(experts=64, ldl=64, k=33) == UNSUPPORTED and call(tokens=1 << 31) == BAD
    assert call(ws=None) == WORKSPACE and call(room=n - 1) == WORKSPACE
    for name, _ in nb._Routing._fields_:
        part = nb._Routing(*[A + 4096 * i for i in range(10)])
        setattr(part, name, None)
        assert call(out=part) == BAD
    grad = lambda grad=E, ldg=16, dg=None: lib.nacho_route_grad(B, 16, 100, 16, nb.F32, 2, 0, C.byref(full), dg, 0.1, grad, ldg, None)
    assert grad(grad=None) == BAD and grad(grad=B) == BAD and grad(ldg=15) == BAD and grad(dg=A + 2) == BAD


def layer(**more):
    base = dict(expert_pos=A, token=A + 4096, n_experts=3, n_slots=50, n_tokens=20, inner=64, outer=96, x=B, ldx=64, w=D, ldw=64,
                w_stride=96 * 64, bias=None, bias_stride=0, act=0, dtype=nb.F32)
    base.update(more)
    return nb._ExpertsLayer(*[base[n] for n, _ in nb._ExpertsLayer._fields_])


def test_experts():
    lib = nb.lib()

    def call(y=E, ldy=96, pre=None, ldpre=0, **more):
        return lib.nacho_experts(C.byref(layer(**more)), y, ldy, pre, ldpre, None)

    assert lib.nacho_experts(None, E, 96, None, 0, None) == BAD
    for wrong in (dict(expert_pos=None), dict(n_experts=0), dict(n_slots=-1), dict(inner=0), dict(outer=0), dict(x=None), dict(ldx=63),
                  dict(w=None), dict(ldw=63), dict(w_stride=96 * 64 - 1), dict(act=4), dict(dtype=nb.F64), dict(y=None), dict(ldy=95),
                  dict(y=B), dict(y=D + 4096), dict(pre=E, ldpre=96), dict(pre=D, ldpre=96), dict(pre=E + (1 << 30), ldpre=95),
                  dict(token=None), dict(bias=A + 2, bias_stride=96), dict(bias=A, bias_stride=95)):
        assert call(**wrong) == BAD, wrong
    assert call(n_experts=70000) == UNSUPPORTED and call(inner=1 << 24, ldx=1 << 24, ldw=1 << 24, w_stride=1 << 40) == UNSUPPORTED
    rc, n = size(lib.nacho_experts_workspace_bytes, C.byref(layer(act=2)))
    assert rc == 0 and n >= 50 * 96 * 4

    def grad(gy=E, ldgy=96, pre=E + (1 << 30), ldpre=96, gx=E + (2 << 30), ldgx=64, gw=E + (3 << 30), ldgw=64, gws=96 * 64, gb=None, gbs=0,
             ws=E + (4 << 30), room=n, **more):
        return lib.nacho_experts_grad(C.byref(layer(**{"act": 2, **more})), gy, ldgy, pre, ldpre, gx, ldgx, gw, ldgw, gws, gb, gbs, ws, room, None)

    for wrong in (dict(gy=None), dict(pre=None), dict(ldgx=63), dict(ldgw=63), dict(gws=5), dict(gx=B), dict(gw=D), dict(gw=E + (2 << 30)),
                  dict(gb=A, gbs=95), dict(gx=E)):
        assert grad(**wrong) == BAD, wrong
    assert grad(ws=None) == WORKSPACE and grad(room=100) == WORKSPACE


def test_combine():
    lib = nb.lib()
    m = lambda **more: teacher(**{"rows": 5, "cols": 12, "stored": 12, **more})

    def call(t=None, y=B, ldy=32, n=32, dtype=nb.F32, residual=None, ldr=0, out=D, ldo=32):
        return lib.nacho_combine(C.byref(t or m()), y, ldy, n, dtype, residual, ldr, out, ldo, None)

    assert call(y=None) == BAD and call(out=None) == BAD and call(ldy=31) == BAD and call(ldo=31) == BAD and call(dtype=nb.F64) == BAD
    assert call(out=B + 128) == BAD and call(residual=D + 128, ldr=32) == BAD and call(residual=D, ldr=33, ldo=32) == BAD and call(n=-1) == BAD
    assert call(m(kinds=(nb.COMPRESSED, nb.COMPRESSED))) == UNSUPPORTED and call(m(pos=None)) == BAD and call(m(crd=None)) == BAD
    grad = lambda y=B, go=D, gy=E, gv=A + (1 << 30): lib.nacho_combine_grad(C.byref(m()), y, 32, 32, nb.F32, go, 32, gy, 32, gv, None)
    assert grad(go=None) == BAD and grad(gy=D) == BAD and grad(y=None) == BAD and grad(gy=B) == BAD and grad(gv=A + 2) == BAD


@pytest.mark.parametrize("call", ["nacho_spmv", "nacho_spmm", "nacho_spadd_k"])
def test_sparse_algebra_still_takes_floats_and_doubles_alone(call):
    with pytest.raises(TypeError):
        import torch
        nb.dtype_code(torch.bfloat16)
    n = C.c_size_t(0)
    t = teacher()
    for dtype in (nb.BF16, nb.F16):
        for op in (nb.OP_SPMV, nb.OP_SPMM, nb.OP_SPADD):
            assert nb.lib().nacho_workspace_bytes(op, C.byref(t), 1, dtype, 8, 0, C.byref(n)) == BAD


def test_sizes_whose_products_pass_64_bits():
    """Stretches longer than any memory still overlap what lies in them."""
    lib = nb.lib()
    most, far = (1 << 31) - 1, 1 << 40
    t = teacher(rows=most, cols=1, stored=10)
    assert lib.nacho_distill(C.byref(t), B, far, nb.F32, None, 1.0, E, E + (1 << 36), B + 4096, 1, None, 0, None) == BAD
    assert lib.nacho_distill_grad(C.byref(t), B, far, nb.F32, None, 1.0, E, B + 4096, far, None) == BAD
    m = teacher(rows=5, cols=most, stored=12)
    assert lib.nacho_combine(C.byref(m), B, far, 32, nb.F32, None, 0, B + (1 << 39), 32, None) == BAD
    # experts that lie on each other
    wide = layer(n_experts=3, outer=(1 << 24) - 1, inner=64, ldw=far, w_stride=1 << 30)
    assert lib.nacho_experts(C.byref(wide), E, 1 << 24, None, 0, None) == BAD
    assert size(lib.nacho_route_workspace_bytes, (1 << 62) + 1, 64, 4)[0] == BAD


# Arrays of a call as (address, bytes); every output of which is put over every other array in turn.
def overlaps(arrays, outputs, call, allowed=()):
    if not torch.cuda.is_available():                        # (where nothing can be launched: the arrays as they are pass)
        assert call() == HIP
    for out in outputs:
        for other, (at, length) in arrays.items():
            if other == out or (out, other) in allowed:
                continue
            for shift in (0, length - 4):                    # its first element there, or its first over the other's last
                assert call(**{out: at + shift}) == BAD, (out, other, shift)


def test_distill_outputs_over_other_arrays():
    lib = nb.lib()
    rows, cols, n = 4, 1 << 20, 10                           # (cut into parts: there is a workspace)
    room = size(lib.nacho_distill_workspace_bytes, rows, cols, nb.F32)[1]
    length = dict(pos=20, crd=40, val=40, logits=rows * cols * 4, weight=16, loss=16, lse=16, grad=rows * cols * 4, ws=room)
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}
    arrays = {name: (base[name], length[name]) for name in length}

    def call(**moved):
        p = {**base, **moved}
        return lib.nacho_distill(C.byref(teacher(rows, cols, n, p["pos"], p["crd"], p["val"])), p["logits"], cols, nb.F32, p["weight"], 1.0, p["loss"],
                                 p["lse"], p["grad"], cols, p["ws"], room, None)

    overlaps(arrays, ("loss", "lse", "grad"), call)
    for name in ("crd", "val", "logits", "weight"):          # (a workspace starts at a multiple of 16 bytes)
        assert call(ws=base[name]) == BAD, name

    def back(**moved):
        p = {**base, **moved}
        return lib.nacho_distill_grad(C.byref(teacher(rows, cols, n, p["pos"], p["crd"], p["val"])), p["logits"], cols, nb.F32, p["weight"], 1.0,
                                      p["lse"], p["grad"], cols, None)

    overlaps({k: v for k, v in arrays.items() if k not in ("loss", "ws")}, ("grad",), back)


def test_route_outputs_over_other_arrays():
    lib = nb.lib()
    tokens, experts, k = 100, 16, 2
    room = size(lib.nacho_route_workspace_bytes, tokens, experts, k)[1]
    names = [n for n, _ in nb._Routing._fields_]
    length = dict(pos=404, expert=800, gate=800, slot=800, expert_pos=68, token=800, counts=64, lse=400, balance=4, routed=4,
                  logits=tokens * experts * 4, keep=tokens, ws=room)
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}
    arrays = {name: (base[name], length[name]) for name in length}

    def call(**moved):
        p = {**base, **moved}
        return lib.nacho_route(p["logits"], experts, tokens, experts, nb.F32, k, 0, p["keep"], C.byref(nb._Routing(*[p[n] for n in names])), p["ws"], room, None)

    overlaps(arrays, names, call)
    for name in names + ["logits", "keep"]:
        assert call(ws=base[name]) == BAD, name
    length.update(grad=tokens * experts * 4, grad_gate=800)
    del length["ws"], length["keep"]
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}

    def back(**moved):
        p = {**base, **moved}
        return lib.nacho_route_grad(p["logits"], experts, tokens, experts, nb.F32, k, 0, C.byref(nb._Routing(*[p[n] for n in names])), p["grad_gate"], 0.1,
                                    p["grad"], experts, None)

    overlaps({name: (base[name], length[name]) for name in length}, ("grad",), back)


def test_experts_outputs_over_other_arrays():
    lib = nb.lib()
    size_of = dict(expert_pos=16, token=200, x=20 * 64 * 4, w=3 * 96 * 64 * 4, bias=3 * 96 * 4, y=50 * 96 * 4, pre=50 * 96 * 4)
    base = {name: (i + 1) << 40 for i, name in enumerate(size_of)}

    def of(p, **more):
        return layer(expert_pos=p["expert_pos"], token=p["token"], x=p["x"], w=p["w"], bias=p.get("bias"), bias_stride=96, **more)

    def call(**moved):
        p = {**base, **moved}
        return lib.nacho_experts(C.byref(of(p)), p["y"], 96, p["pre"], 96, None)

    overlaps({n: (base[n], size_of[n]) for n in size_of}, ("y", "pre"), call)
    room = size(lib.nacho_experts_workspace_bytes, C.byref(layer(act=2)))[1]
    del size_of["bias"], size_of["y"]
    size_of.update(grad_y=50 * 96 * 4, grad_x=50 * 64 * 4, grad_w=3 * 96 * 64 * 4, grad_bias=3 * 96 * 4, ws=room)
    base = {name: (i + 1) << 40 for i, name in enumerate(size_of)}

    def back(**moved):
        p = {**base, **moved}
        return lib.nacho_experts_grad(C.byref(of(p, act=2)), p["grad_y"], 96, p["pre"], 96, p["grad_x"], 64, p["grad_w"], 64, 96 * 64, p["grad_bias"], 96,
                                      p["ws"], room, None)

    overlaps({n: (base[n], size_of[n]) for n in size_of}, ("grad_x", "grad_w", "grad_bias"), back)
    for name in size_of:
        if name != "ws":
            assert back(ws=base[name]) == BAD, name


def test_combine_outputs_over_other_arrays():
    lib = nb.lib()
    length = dict(pos=24, slot=48, gate=48, y=12 * 32 * 4, residual=5 * 32 * 4, out=5 * 32 * 4)
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}

    def call(**moved):
        p = {**base, **moved}
        return lib.nacho_combine(C.byref(teacher(5, 12, 12, p["pos"], p["slot"], p["gate"])), p["y"], 32, 32, nb.F32, p["residual"], 32, p["out"], 32, None)

    overlaps({n: (base[n], length[n]) for n in length}, ("out",), call, allowed=(("out", "residual"),))
    assert call(out=base["residual"] + 128) == BAD           # (in place is the residual itself alone)
    length = dict(pos=24, slot=48, gate=48, y=12 * 32 * 4, grad_out=5 * 32 * 4, grad_y=12 * 32 * 4, grad_val=48)
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}

    def back(**moved):
        p = {**base, **moved}
        return lib.nacho_combine_grad(C.byref(teacher(5, 12, 12, p["pos"], p["slot"], p["gate"])), p["y"], 32, 32, nb.F32, p["grad_out"], 32, p["grad_y"], 32,
                                      p["grad_val"], None)

    overlaps({n: (base[n], length[n]) for n in length}, ("grad_y", "grad_val"), back)


def test_distill_arrays_between_elements():
    """Positions, weights, losses and lse that start between two elements."""
    lib = nb.lib()

    def call(pos=A, weight=D, loss=E, lse=E + 4096):
        return lib.nacho_distill(C.byref(teacher(pos=pos)), B, 100, nb.F32, weight, 1.0, loss, lse, None, 0, None, 0, None)

    def back(pos=A, weight=D, lse=E):
        return lib.nacho_distill_grad(C.byref(teacher(pos=pos)), B, 100, nb.F32, weight, 1.0, lse, E + (1 << 30), 100, None)

    for f in (call, back):
        assert f(pos=A + 2) == BAD and f(weight=D + 1) == BAD and f(lse=E + 4098) == BAD
    assert call(loss=E + 2) == BAD
