"""What the Python side of the cross entropy, the rows in 8 bits and the layer of single steps refuses and makes before the library is
called (the library's calls are replaced, nothing is launched, no GPU)."""
import pytest
import torch

from paper_2604_17198_amd import binding as nb
from test_model_binding import calls, ints  # noqa: F401


def step_args(dtype=torch.float32):
    return dict(x=torch.zeros((3, 16), dtype=dtype), logits=torch.zeros((3, 5), dtype=dtype), top_k=2, up=torch.zeros((5, 24, 16), dtype=dtype),
                down=torch.zeros((5, 20, 24), dtype=dtype))


def test_step_refuses(calls):  # noqa: F811
    z = torch.zeros
    good = step_args()
    for wrong in (dict(x=z(3, 17)), dict(x=z(3, 2, 16)), dict(logits=z(3, 6)), dict(logits=z(2, 5)), dict(logits=z((3, 5), dtype=torch.bfloat16)), dict(up=z(24, 16)),
                  dict(up=z(5, 24, 15)), dict(up=z((5, 24, 16), dtype=torch.float16)), dict(down=z(4, 20, 24)), dict(down=z(5, 20, 23)), dict(down=z(5, 24, 20).transpose(1, 2)),
                  dict(up=z(5, 1, 16).expand(5, 24, 16)), dict(gate=z(5, 24, 17)), dict(gate_bias=z(5, 24)),
                  dict(gate=z(5, 24, 16), gate_bias=z(5, 23)), dict(up_bias=z(5, 23)), dict(up_bias=z((5, 24), dtype=torch.float64)), dict(down_bias=z(4, 20)), dict(residual=z(3, 21)),
                  dict(residual=z((3, 20), dtype=torch.bfloat16)), dict(out=z(2, 20)), dict(keep=z(3)), dict(keep=z(2, dtype=torch.bool)), dict(act="tanh"),
                  dict(ws=torch.empty(1 << 20, dtype=torch.uint8, device="meta")), dict(x=torch.empty((3, 16), device="meta"))):
        with pytest.raises(ValueError):
            nb.nacho_experts_step(**{**good, **wrong})
    assert "nacho_experts_step" not in calls
    with pytest.raises(TypeError):
        nb.nacho_experts_step(**step_args(torch.float64))
    out = nb.nacho_experts_step(**good, gate=z(5, 24, 16), gate_bias=z(5, 24), up_bias=z(5, 24), down_bias=z(5, 20), residual=z(3, 20), keep=z(3, dtype=torch.bool))
    assert out.shape == (3, 20) and out.dtype is torch.float32 and calls[-1] == "nacho_experts_step"


@pytest.mark.parametrize("top_k", [0, -1, 6, 2 ** 32 + 2, -2 ** 32 + 2, 2 ** 64 + 1])
def test_numbers_of_experts_that_there_are_not(calls, top_k):  # noqa: F811
    """Not one of them is taken for its lowest 32 bits."""
    with pytest.raises(ValueError):
        nb.nacho_experts_step(**{**step_args(), "top_k": top_k})
    assert "nacho_experts_step" not in calls


def test_xent_refuses(calls):  # noqa: F811
    z = torch.zeros
    good = dict(x=z(4, 16), head=z(30, 16), label=z(4, dtype=torch.int64))
    for wrong in (dict(x=z(4, 15)), dict(x=z(16)), dict(head=z((30, 16), dtype=torch.bfloat16)), dict(head=z(30, 32)[:, ::2]), dict(label=z(5, dtype=torch.int64)),
                  dict(label=z(4)), dict(label=z(4, dtype=torch.int16)), dict(label=z(8, dtype=torch.int64)[::2]), dict(weight=z(3)), dict(weight=z(4, dtype=torch.float64)),
                  dict(weight=torch.empty(4, device="meta"))):
        with pytest.raises(ValueError):
            nb.nacho_xent(**{**good, **wrong})
        with pytest.raises(ValueError):
            nb.nacho_xent_grad(**{**good, **wrong}, lse=z(4))
    for wrong in (dict(loss=z(3)), dict(lse=z(4, dtype=torch.float64)), dict(ws=torch.zeros(1 << 20, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            nb.nacho_xent(**good, **wrong)
    for wrong in (dict(lse=z(3)), dict(lse=z(4), grad_x=z(4, 15)), dict(lse=z(4), grad_head=z(29, 16)), dict(lse=z(4), grad_head=z((30, 16), dtype=torch.float16))):
        with pytest.raises(ValueError):
            nb.nacho_xent_grad(**good, **wrong)
    assert "nacho_xent" not in calls and "nacho_xent_grad" not in calls


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_results_do_not_take_the_default_type(calls, default):  # noqa: F811
    before = torch.get_default_dtype()
    try:
        torch.set_default_dtype(default)
        x, head, label = torch.zeros((4, 16), dtype=torch.float16), torch.zeros((30, 16), dtype=torch.float16), torch.zeros(4, dtype=torch.int32)
        loss, lse = nb.nacho_xent(x, head, label)
        gx, gh = nb.nacho_xent_grad(x, head, label, lse)
        kept = nb.nacho_keep8(x)
        assert loss.dtype is torch.float32 and lse.dtype is torch.float32 and gx.dtype is torch.float16 and gh.dtype is torch.float16
        assert kept.codes.dtype is torch.int8 and kept.exponent.dtype is torch.uint8 and nb.nacho_restore8(kept).dtype is torch.float32
    finally:
        torch.set_default_dtype(before)


def test_rows_in_8_bits(calls):  # noqa: F811
    z = torch.zeros
    codes, exponent = z((4, 40), dtype=torch.int8), z((4, 2), dtype=torch.uint8)
    for c, e in ((codes.float(), exponent), (codes, exponent.to(torch.int8)), (codes, exponent[:3]), (codes, exponent[:, :1]), (codes.T, exponent), (codes[0], exponent),
                 (codes, torch.empty((4, 2), dtype=torch.uint8, device="meta"))):
        with pytest.raises(ValueError):
            nb.Kept8(c, e)
    kept = nb.Kept8(codes, exponent)
    assert nb.Kept8.empty(4, 40, codes.device).codes.stride() == (48, 1) and kept.shape == (4, 40)
    for f in (lambda: nb.nacho_keep8(z(4, 41), out=kept), lambda: nb.nacho_keep8(z(3, 40), out=kept), lambda: nb.nacho_restore8(kept, out=z(4, 41)),
              lambda: nb.nacho_keep8(z(4, 80)[:, ::2])):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        nb.nacho_keep8(z((4, 40), dtype=torch.float64))
    with pytest.raises(TypeError):
        nb.nacho_restore8(kept, torch.float64)
    x, w, bounds, gy = z(4, 40), z(2, 24, 40), ints(0, 1, 4), z(4, 24)
    pre = nb.Kept8.empty(4, 24, x.device)
    for f in (lambda: nb.nacho_experts(kept, w, bounds), lambda: nb.nacho_experts(x, w, bounds, pre=kept), lambda: nb.nacho_experts_grad(gy, kept, z(2, 24, 39), bounds),
              lambda: nb.nacho_experts_grad(gy, kept, w, bounds, pre=kept), lambda: nb.nacho_experts_grad(gy.half(), kept, w, bounds, pre=pre)):
        with pytest.raises(ValueError):
            f()
    calls.clear()
    nb.nacho_experts(x, w, bounds, pre=pre)
    nb.nacho_experts_grad(gy, kept, w, bounds, pre=pre)
    nb.nacho_experts_grad(gy, x, w, bounds, act="silu", pre=pre)
    nb.nacho_experts_grad(gy, kept, w, bounds, act="silu", pre=z(4, 24))
    nb.nacho_experts_grad(gy, x, w, bounds, act="silu", pre=z(4, 24))
    assert [c for c in calls if not c.endswith("_bytes")] == ["nacho_experts_keep8"] + ["nacho_experts_keep8_grad"] * 3 + ["nacho_experts_grad"]


def test_arrays_of_kept_rows_stay_those_of_the_descriptor():
    kept = nb.Kept8(torch.zeros((4, 40), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8))
    for name in ("codes", "exponent"):
        with pytest.raises(AttributeError):
            setattr(kept, name, getattr(kept, name).clone())
    assert kept.c.code == kept.codes.data_ptr() and kept.c.exponent == kept.exponent.data_ptr()


def test_host_tensors_are_refused():
    z = torch.zeros
    kept = nb.Kept8(z((4, 40), dtype=torch.int8), z((4, 2), dtype=torch.uint8))
    for f in (lambda: nb.nacho_xent(z(4, 16), z(30, 16), z(4, dtype=torch.int64)), lambda: nb.nacho_xent_grad(z(4, 16), z(30, 16), z(4, dtype=torch.int64), z(4)),
              lambda: nb.nacho_keep8(z(4, 40)), lambda: nb.nacho_restore8(kept), lambda: nb.nacho_experts_step(**step_args()),
              lambda: nb.nacho_experts_grad(z(4, 24), kept, z(2, 24, 40), ints(0, 1, 4))):
        with pytest.raises(ValueError):
            f()
