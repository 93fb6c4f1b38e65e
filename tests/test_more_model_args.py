"""What the cross entropy, the rows in 8 bits and the layer of single steps refuse, asked of the built library with made-up addresses
(nothing is launched, no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_17198_amd import binding as nb
from test_model_args import BAD, HIP, UNSUPPORTED, WORKSPACE, overlaps, size

A, B, D, E = 1 << 40, 2 << 40, 3 << 40, 4 << 40              # addresses far apart
OK = 0 if torch.cuda.is_available() else HIP


def xent(**more):
    base = dict(n_rows=50, vocabulary=300, inner=64, x=A, ldx=64, head=B, ldh=64, label=D, weight=D + 4096, label_bytes=8, dtype=nb.F32)
    base.update(more)
    return nb._XentLayer(*[base[n] for n, _ in nb._XentLayer._fields_])


WRONG_XENT = [dict(n_rows=-1), dict(n_rows=1 << 31), dict(vocabulary=0), dict(inner=0), dict(x=None), dict(ldx=63), dict(x=A + 2), dict(head=None), dict(ldh=63),
              dict(label=None), dict(label=D + 4), dict(weight=D + 2), dict(label_bytes=2), dict(label_bytes=0), dict(dtype=nb.F64)]


def test_xent():
    lib = nb.lib()
    rc, n = size(lib.nacho_xent_workspace_bytes, C.byref(xent()))

    def call(loss=E, lse=E + 4096, ws=E + (1 << 30), room=n, **more):
        return lib.nacho_xent(C.byref(xent(**more)), loss, lse, ws, room, None)

    assert rc == 0 and n >= 50 * 4 * 3
    for wrong in WRONG_XENT + [dict(loss=None), dict(lse=None), dict(loss=E + 2), dict(lse=E + 4098)]:
        assert call(**wrong) == BAD, wrong
    assert call(vocabulary=1 << 24) == UNSUPPORTED and call(inner=1 << 24, ldx=1 << 24, ldh=1 << 24) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(room=n - 1) == WORKSPACE and call(ws=E + (1 << 30) + 8) == WORKSPACE
    assert lib.nacho_xent(None, E, E, E, n, None) == BAD and lib.nacho_xent_workspace_bytes(C.byref(xent()), None) == BAD
    assert size(lib.nacho_xent_workspace_bytes, C.byref(xent(dtype=nb.F64)))[0] == BAD


def test_xent_grad():
    lib = nb.lib()
    rc, n = size(lib.nacho_xent_grad_workspace_bytes, C.byref(xent()))

    def call(lse=E, gx=E + (1 << 30), ldgx=64, gh=E + (2 << 30), ldgh=64, ws=E + (3 << 30), room=n, **more):
        return lib.nacho_xent_grad(C.byref(xent(**more)), lse, gx, ldgx, gh, ldgh, ws, room, None)

    assert rc == 0 and n >= 50 * 300 * 4
    for wrong in WRONG_XENT + [dict(lse=None), dict(lse=E + 2), dict(ldgx=63), dict(ldgh=63), dict(gx=E + 2), dict(gh=B)]:
        assert call(**wrong) == BAD, wrong
    assert call(ws=None) == WORKSPACE and call(room=n - 1) == WORKSPACE
    # g of a piece of the vocabulary takes 256 MiB at most, whatever the sizes
    large = size(lib.nacho_xent_grad_workspace_bytes, C.byref(xent(n_rows=16_384, vocabulary=200_000, inner=2048, ldx=2048, ldh=2048, dtype=nb.BF16)))[1]
    assert large < (256 << 20) + 4 * 16_384 * 2048 * 4 + (1 << 21)
    assert call(gx=None, gh=None) == 0                       # (nothing is wanted, nothing launched)


def kept(code=E, ldc=64, exponent=E + (1 << 30), lde=2):
    return nb._Kept(code, ldc, exponent, lde)


def test_kept():
    lib = nb.lib()

    def keep(x=A, ldx=64, rows=10, cols=64, dtype=nb.BF16, k=None):
        return lib.nacho_keep8(x, ldx, rows, cols, dtype, C.byref(k or kept()), None)

    def restore(out=A, ldo=64, rows=10, cols=64, dtype=nb.BF16, k=None):
        return lib.nacho_restore8(C.byref(k or kept()), rows, cols, dtype, out, ldo, None)

    for f, name, ld in ((keep, "x", "ldx"), (restore, "out", "ldo")):
        for wrong in ({name: None}, {name: A + 1}, {ld: 63}, dict(rows=-1), dict(rows=1 << 31), dict(cols=-1), dict(cols=1 << 31), dict(dtype=nb.F64),
                      dict(k=kept(code=None)), dict(k=kept(ldc=63)), dict(k=kept(exponent=None)), dict(k=kept(lde=1)), {name: E}, {name: E + (1 << 30)}):
            assert f(**wrong) == BAD, (f, wrong)
    assert lib.nacho_keep8(A, 64, 10, 64, nb.BF16, None, None) == BAD and lib.nacho_restore8(None, 10, 64, nb.BF16, A, 64, None) == BAD
    assert keep(k=kept(exponent=E + 640 - 1)) == BAD         # codes over exponents
    if not torch.cuda.is_available():
        assert keep() == HIP and restore() == HIP


def layer(**more):
    base = dict(expert_pos=A, token=A + 4096, n_experts=3, n_slots=50, n_tokens=20, inner=64, outer=96, x=B, ldx=64, w=D, ldw=64,
                w_stride=96 * 64, bias=None, bias_stride=0, act=2, dtype=nb.F32)
    base.update(more)
    return nb._ExpertsLayer(*[base[n] for n, _ in nb._ExpertsLayer._fields_])


def test_experts_that_keep_their_rows():
    lib = nb.lib()
    pre = kept(E, 96, E + (1 << 30), 3)
    assert lib.nacho_experts_keep8(C.byref(layer()), E + (2 << 30), 96, None, None) == BAD
    for k in (kept(E, 95, E + (1 << 30), 3), kept(E, 96, E + (1 << 30), 2), kept(None, 96, E, 3), kept(B, 96, E, 3), kept(E, 96, E + 50 * 96 - 1, 3)):
        assert lib.nacho_experts_keep8(C.byref(layer()), E + (2 << 30), 96, C.byref(k), None) == BAD
    assert lib.nacho_experts_keep8(C.byref(layer(x=None)), E + (2 << 30), 96, C.byref(pre), None) == BAD
    rc, n = size(lib.nacho_experts_keep8_workspace_bytes, C.byref(layer()))
    assert rc == 0 and n >= 50 * 96 * 4 + 20 * 64 * 4

    def grad(x8=None, gy=A + (1 << 30), pre16=None, pre8=pre, gx=A + (2 << 30), gw=A + (3 << 30), ws=A + (4 << 30), room=n, **more):
        by = lambda k: C.byref(k) if k is not None else None
        return lib.nacho_experts_keep8_grad(C.byref(layer(**more)), by(x8), gy, 96, pre16, 96, by(pre8), gx, 64, gw, 64, 96 * 64, None, 0, ws, room, None)

    x8 = kept(E + (2 << 30), 64, E + (3 << 30), 2)
    for wrong in (dict(gy=None), dict(x=None), dict(pre8=None), dict(x8=kept(E, 63, E + 4096, 2)), dict(x8=kept(E, 64, None, 2)), dict(gx=E), dict(gw=E + (2 << 30), x8=x8),
                  dict(gw=E + (3 << 30), x8=x8), dict(pre8=kept(E, 95, E, 3))):
        assert grad(**wrong) == BAD, wrong
    assert grad(ws=None) == WORKSPACE and grad(x8=x8, room=100) == WORKSPACE
    if not torch.cuda.is_available():
        assert grad(x8=x8, x=None) == HIP                    # (x is not read)


def step(**more):
    base = dict(n_tokens=5, n_experts=8, inner=64, hidden=96, outer=80, logits=A, ldl=8, keep=A + 4096, x=A + 8192, ldx=64, up=dict(), gate=dict(w=B + (1 << 38)),
                down=dict(w=B + (2 << 38)), residual=D, ldr=80, out=E, ldo=80, top_k=2, normalise=1, act=3, dtype=nb.F32)
    base.update(more)
    rows = dict(up=(96, 64), gate=(96, 64), down=(80, 96))
    for name, (r, c) in rows.items():
        d = dict(w=B, ld=c, stride=r * c, bias=None, bias_stride=0)
        d.update(base[name])
        base[name] = nb._Dense(*[d[n] for n, _ in nb._Dense._fields_])
    return nb._StepLayer(*[base[n] for n, _ in nb._StepLayer._fields_])


def test_step():
    lib = nb.lib()
    rc, n = size(lib.nacho_experts_step_workspace_bytes, C.byref(step()))
    assert rc == 0 and n >= 5 * 2 * 96 * 4

    def call(ws=E + (1 << 30), room=n, **more):
        return lib.nacho_experts_step(C.byref(step(**more)), ws, room, None)

    for wrong in (dict(n_tokens=-1), dict(n_experts=0), dict(inner=0), dict(hidden=0), dict(outer=0), dict(top_k=0), dict(top_k=9), dict(act=4), dict(dtype=nb.F64),
                  dict(logits=None), dict(ldl=7), dict(x=None), dict(ldx=63), dict(out=None), dict(ldo=79), dict(ldr=79), dict(up=dict(w=None)), dict(up=dict(ld=63)),
                  dict(up=dict(stride=96 * 64 - 1)), dict(up=dict(bias=A + 2, bias_stride=96)), dict(up=dict(bias=A, bias_stride=95)), dict(gate=dict(ld=63)),
                  dict(gate=dict(w=None, bias=A)), dict(down=dict(w=None)), dict(down=dict(ld=95)), dict(down=dict(stride=1)), dict(down=dict(bias=A, bias_stride=79)),
                  dict(out=A), dict(out=A + 8192), dict(out=B), dict(out=B + (1 << 38)), dict(out=B + (2 << 38)), dict(out=D + 4), dict(out=D, ldo=81),
                  dict(out=A + 4096)):
        assert call(**wrong) == BAD, wrong
    for more in (dict(n_tokens=65), dict(n_experts=1025, ldl=1025), dict(top_k=33, n_experts=64, ldl=64), dict(inner=1 << 24), dict(hidden=1 << 24), dict(outer=1 << 24)):
        assert call(**more) == UNSUPPORTED, more
    assert call(ws=None) == WORKSPACE and call(room=n - 1) == WORKSPACE and lib.nacho_experts_step(None, E, n, None) == BAD
    assert call(ws=B) == BAD and call(ws=D) == BAD
    assert call(n_tokens=0) == 0
    if not torch.cuda.is_available():
        assert call(out=D) == HIP and call(gate=dict(w=None)) == HIP and call() == HIP


def test_outputs_over_other_arrays():
    lib = nb.lib()
    length = dict(x=50 * 64 * 4, head=300 * 64 * 4, label=400, weight=200, loss=200, lse=200)
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}
    n = size(lib.nacho_xent_workspace_bytes, C.byref(xent()))[1]

    def call(**moved):
        p = {**base, **moved}
        return lib.nacho_xent(C.byref(xent(**{k: p[k] for k in ("x", "head", "label", "weight")})), p["loss"], p["lse"], 1 << 50, n, None)

    overlaps({k: (base[k], length[k]) for k in length}, ("loss", "lse"), call)
    for name in length:
        p = dict(base)
        assert lib.nacho_xent(C.byref(xent(**{k: p[k] for k in ("x", "head", "label", "weight")})), p["loss"], p["lse"], p[name], n, None) == BAD
    length.update(gx=50 * 64 * 4, gh=300 * 64 * 4)
    del length["loss"]
    base = {name: (i + 1) << 40 for i, name in enumerate(length)}
    room = size(lib.nacho_xent_grad_workspace_bytes, C.byref(xent()))[1]

    def back(ws=1 << 50, **moved):
        p = {**base, **moved}
        return lib.nacho_xent_grad(C.byref(xent(**{k: p[k] for k in ("x", "head", "label", "weight")})), p["lse"], p["gx"], 64, p["gh"], 64, ws, room, None)

    overlaps({k: (base[k], length[k]) for k in length}, ("gx", "gh"), back)
    for name in length:
        assert back(ws=base[name]) == BAD, name


def test_sizes_whose_products_pass_64_bits():
    """Rows and leading dimensions at their limits: refused or taken, never wrapped around."""
    lib = nb.lib()
    most, far = (1 << 31) - 1, 1 << 40
    assert lib.nacho_keep8(A, far, most, 32, nb.BF16, C.byref(kept(A + (1 << 50), far, E, far)), None) == BAD
    assert lib.nacho_restore8(C.byref(kept(A, far, E, far)), most, 32, nb.BF16, A + 4096, far, None) == BAD
    rc, n = size(lib.nacho_xent_grad_workspace_bytes, C.byref(xent(n_rows=most, vocabulary=2000, ldx=far, ldh=far)))
    assert rc == 0 and n > 256 * most * 4
    assert size(lib.nacho_xent_grad_workspace_bytes, C.byref(xent(n_rows=most, vocabulary=(1 << 24) - 1, ldx=far, ldh=far)))[0] == UNSUPPORTED
    assert size(lib.nacho_xent_workspace_bytes, C.byref(xent(vocabulary=(1 << 24) - 1, inner=(1 << 24) - 1, ldx=far, ldh=far)))[0] == UNSUPPORTED
    assert lib.nacho_xent_grad(C.byref(xent(n_rows=most, ldx=far)), E, B, 64, None, 0, E + (1 << 45), 1 << 62, None) == BAD


@pytest.mark.parametrize("inner", [8, 96, 1024, 5000, 16_384])
@pytest.mark.parametrize("rows", [1, 16, 17, 300, 511, 4096, 32_767, 32_768, 300_000, 1_100_000])
@pytest.mark.parametrize("vocabulary", [1, 1000, 32_768, 100_003, 1_000_000])
@pytest.mark.parametrize("dtype", [nb.F32, nb.BF16])
def test_workspaces_are_what_the_header_says(rows, vocabulary, inner, dtype):
    lib = nb.lib()
    elem, whole = (4 if dtype == nb.F32 else 2), -(-vocabulary // 8) * 8
    at = xent(n_rows=rows, vocabulary=vocabulary, inner=inner, ldx=inner, ldh=inner, dtype=dtype)
    rc, loss = size(lib.nacho_xent_workspace_bytes, C.byref(at))
    narrowest = 128 if elem == 2 else 64 if -(-rows // 16) * -(-vocabulary // 32) > 1024 else 32
    parts = -(-vocabulary // narrowest)
    if rows <= 16:
        parts = max(parts, min(1024, -(-vocabulary // (64 if vocabulary < 24_576 else 128))))      # (four wavefronts of 16 or 32 words)
    lists = 40 * rows + (1 << 15)
    assert rc == 0 and 8 * rows * parts <= loss <= 8 * rows * parts + lists
    rc, grad = size(lib.nacho_xent_grad_workspace_bytes, C.byref(at))
    g = min(rows * whole * elem, max(256 << 20, rows * 256 * elem))
    assert rc == 0 and grad <= g + max(256 << 20, rows * inner * 4) + lists


@pytest.mark.parametrize("rows", [1, 64, 65, 3000, 100_000])
@pytest.mark.parametrize("vocabulary", [1, 255, 256, 32_767, 32_768, 200_001])
@pytest.mark.parametrize("dtype", [nb.F32, nb.BF16])
def test_workspaces_grow_with_rows(rows, vocabulary, dtype):
    """(the statistics of every tile there can be; g of a piece in whole words of 8)"""
    lib = nb.lib()
    elem = 4 if dtype == nb.F32 else 2
    a = size(lib.nacho_xent_workspace_bytes, C.byref(xent(n_rows=rows, vocabulary=vocabulary, dtype=dtype)))[1]
    assert a >= rows * 8 * -(-vocabulary // 256)
    g = size(lib.nacho_xent_grad_workspace_bytes, C.byref(xent(n_rows=rows, vocabulary=vocabulary, dtype=dtype)))[1]
    assert g >= min(rows * vocabulary * elem, rows * 256 * elem)
