"""Tensors of another type, or too short, in the calls of rotary positions, gated norms and 8-bit integer linear layers: refused by the binding before anything reads or writes
them (no GPU is touched here: the tensors lie in host memory, which is refused as well, after their types and sizes)."""
import pytest
import torch

import paper_2508_17756_amd as sg

TOKENS, HEADS, D, ROWS, C = 24, 4, 64, 6, 256
F32, BF16, I8, E4M3 = torch.float32, torch.bfloat16, torch.int8, torch.float8_e4m3fn
no_device = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="calls that are not refused would be launched")


def _many(kind, *shape, n=2):
    return [torch.zeros(shape, dtype=kind) for _ in range(n)]


class OnDevice(torch.Tensor):
    """Host memory that says it is the device's, for what is looked at behind that."""
    is_cuda = True


def _device(t):
    return t.as_subclass(OnDevice)


def _rotary(dtype, **kw):
    kind = {"f32": F32, "bf16": BF16}[dtype]
    p = sg.make_rotary_problem((2, 3, 4), HEADS, D, dtype, (16, 24, 24))
    a = dict(q=_many(kind, HEADS, TOKENS, D), q_out=_many(kind, HEADS, TOKENS, D), k=_many(kind, HEADS, TOKENS, D), k_out=_many(kind, HEADS, TOKENS, D),
             frequencies=_device(torch.zeros(32, dtype=torch.float64)), origin=[(0, 0, 0)] * 2, q_weight=_device(torch.ones(D, dtype=kind)), k_weight=None)
    a.update(kw)
    return sg.sg_tile_rotary(p, a.pop("q"), a.pop("q_out"), a.pop("frequencies"), **a)


@pytest.mark.parametrize("dtype, kind, other", [("f32", F32, BF16), ("bf16", BF16, F32), ("bf16", BF16, torch.float16)])
def test_rotary_takes_its_type_only(dtype, kind, other):
    for name in ("q", "q_out", "k", "k_out"):
        mixed = [torch.zeros((HEADS, TOKENS, D), dtype=k) for k in (kind, other)]
        with pytest.raises(TypeError, match=name):
            _rotary(dtype, **{name: mixed})
        with pytest.raises(ValueError):
            _rotary(dtype, **{name: mixed[:1]})
    for name in ("q_weight", "k_weight"):
        with pytest.raises(TypeError, match=name):
            _rotary(dtype, **{name: _device(torch.ones(D, dtype=other))})
        with pytest.raises(ValueError, match=name):
            _rotary(dtype, **{name: _device(torch.ones(D - 1, dtype=kind))})
        with pytest.raises(ValueError, match=name):
            _rotary(dtype, **{name: _device(torch.ones(2 * D, dtype=kind))[::2]})
        with pytest.raises(ValueError, match=name):
            _rotary(dtype, **{name: torch.ones(D, dtype=kind)})


def _norm(dtype="bf16", fields=None, more=None, **kw):
    kind = {"f32": F32, "bf16": BF16}[dtype]
    p = sg.make_gated_norm_problem(ROWS, C, dtype, **{"post_norm": "rms", **(more or {})})
    for name, value in (fields or {}).items():
        setattr(p, name, value)
    mod = F32 if p.mod_dtype == sg.SG_F32 else kind
    vectors = -(-ROWS // p.mod_rows) if p.mod_rows else 1
    vec = lambda: [_device(t) for t in _many(mod, vectors, C)]   # noqa: E731
    out = {sg.SG_F8_E4M3: E4M3, sg.SG_I8: I8}.get(p.out_dtype, kind)
    groups = C // p.scale_group if p.scale_group else 1
    a = dict(x=_many(kind, ROWS, C), out=_many(out, ROWS, C), residual=_many(kind, ROWS, C), gate=vec(), scale=vec(), shift=vec(), sum_out=_many(kind, ROWS, C),
             post_weight=_device(torch.ones(C, dtype=kind)), weight=_device(torch.ones(C, dtype=kind)),
             out_scale=[_device(t) for t in _many(F32, ROWS, groups)] if out in (E4M3, I8) else None)
    a.update(kw)
    return sg.sg_tile_gated_norm(p, a.pop("x"), a.pop("out"), **a)


@pytest.mark.parametrize("dtype, kind, other", [("f32", F32, BF16), ("bf16", BF16, F32)])
def test_norms_take_their_types_only(dtype, kind, other):
    for name in ("x", "out", "residual", "sum_out"):
        with pytest.raises(TypeError, match=name):
            _norm(dtype, **{name: [torch.zeros((ROWS, C), dtype=k) for k in (kind, other)]})
    for name in ("weight", "post_weight"):
        with pytest.raises(TypeError, match=name):
            _norm(dtype, **{name: _device(torch.ones(C, dtype=other))})
        with pytest.raises(ValueError, match=name):
            _norm(dtype, **{name: _device(torch.ones(C - 8, dtype=kind))})


@pytest.mark.parametrize("dtype, mods, right, wrong", [("bf16", None, BF16, F32), ("bf16", "f32", F32, BF16), ("f32", None, F32, BF16)])
@pytest.mark.parametrize("name", ["gate", "scale", "shift"])
def test_vectors_are_of_the_type_and_number_that_the_problem_says(dtype, mods, right, wrong, name):
    more = {"mod_dtype": mods, "mod_rows": 4}
    with pytest.raises(TypeError, match=name):
        _norm(dtype, more=more, **{name: [_device(t) for t in _many(wrong, 2, C)]})
    with pytest.raises(ValueError, match=name):   # six rows, four to a vector: two vectors
        _norm(dtype, more=more, **{name: [_device(t) for t in _many(right, 1, C)]})
    with pytest.raises(ValueError, match=name):
        _norm(dtype, more={**more, "mod_rows": 0}, **{name: [_device(t) for t in _many(right, 1, C - 8)]})
    with pytest.raises(ValueError, match=name):
        _norm(dtype, more=more, **{name: _many(right, 2, C)})


@pytest.mark.parametrize("out, wrong", [("e4m3", (I8, BF16, F32, torch.float8_e5m2)), ("int8", (E4M3, BF16, torch.uint8))])
@pytest.mark.parametrize("group", [0, 128])
def test_eight_bits_and_their_scales(out, wrong, group):
    more = {"out_dtype": out, "scale_group": group}
    for kind in wrong:
        with pytest.raises(TypeError, match="out"):
            _norm(more=more, out=_many(kind, ROWS, C))
    for kind in (torch.float16, BF16, torch.float64):
        with pytest.raises(TypeError, match="out_scale"):
            _norm(more=more, out_scale=[_device(t) for t in _many(kind, ROWS, 2)])
    short = ROWS * (C // group if group else 1) - 1
    with pytest.raises(ValueError, match="out_scale"):
        _norm(more=more, out_scale=[_device(t) for t in _many(F32, short)])
    with pytest.raises(ValueError, match="out_scale"):
        _norm(more=more, out_scale=[_device(t)[:, :2] for t in _many(F32, ROWS, 4)])


def _linear(dtype="bf16", **kw):
    kind = {"f32": F32, "bf16": BF16}[dtype]
    p = sg.make_int8_linear_problem(ROWS, 64, 40, dtype)
    a = dict(x=_many(I8, ROWS, 64), x_scale=[_device(t) for t in _many(F32, ROWS)], w=_device(torch.zeros((40, 64), dtype=I8)), w_scale=_device(torch.ones(40)),
             out=_many(kind, ROWS, 40), bias=_device(torch.zeros(40, dtype=kind)))
    a.update(kw)
    return sg.sg_tile_int8_linear(p, *(a.pop(n) for n in ("x", "x_scale", "w", "w_scale", "out")), **a)


@pytest.mark.parametrize("dtype, kind, other", [("f32", F32, BF16), ("bf16", BF16, F32)])
def test_linear_takes_its_types_only(dtype, kind, other):
    with pytest.raises(TypeError, match="out"):
        _linear(dtype, out=[torch.zeros((ROWS, 40), dtype=k) for k in (kind, other)])
    with pytest.raises(TypeError, match="bias"):
        _linear(dtype, bias=_device(torch.zeros(40, dtype=other)))
    with pytest.raises(ValueError, match="bias"):
        _linear(dtype, bias=_device(torch.zeros(39, dtype=kind)))
    with pytest.raises(ValueError, match="bias"):
        _linear(dtype, bias=torch.zeros(40, dtype=kind))
    with pytest.raises(TypeError, match="x"):
        _linear(dtype, x=_many(torch.uint8, ROWS, 64))
    with pytest.raises(TypeError, match="w"):
        _linear(dtype, w=_device(torch.zeros((40, 64), dtype=torch.uint8)))
    with pytest.raises(ValueError, match="w"):
        _linear(dtype, w=_device(torch.zeros((39, 64), dtype=I8)))


@no_device
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_right_ones_pass(dtype):
    """(They end with the missing device's error, or at its lack.)"""
    calls = [lambda: _rotary(dtype), lambda: _norm(dtype), lambda: _norm(dtype, more={"mod_dtype": "f32", "mod_rows": 4}), lambda: _linear(dtype),
             lambda: _norm(dtype, more={"mod_rows": 4}, gate=[_device(torch.zeros((2, C + 16), dtype={"f32": F32, "bf16": BF16}[dtype]))[:, :C]] * 2, fields={"mod_stride": C + 16})]
    calls += [lambda o=o, g=g: _norm(dtype, more={"out_dtype": o, "scale_group": g}) for o in ("e4m3", "int8") for g in (0, 128)]
    calls += [lambda: _norm(dtype, more={"out_dtype": "e4m3"}, out=_many(torch.uint8, ROWS, C))]   # its bits
    for call in calls:
        with pytest.raises((sg.SgError, RuntimeError, AssertionError)) as e:
            call()
        assert not isinstance(e.value, (TypeError, ValueError)) and (not isinstance(e.value, sg.SgError) or "-4" in str(e.value) or e.value.status == sg.SG_ERR_HIP)
