"""Argument checks of rotary positions, gated norms and 8-bit integer linear layers, and the rotary frequencies, on the host: a call that cannot be made is
refused before anything is launched (no GPU is touched here)."""
import ctypes
import math

import pytest
import torch

import paper_2508_17756_amd as sg

GOOD = 0x10000   # an aligned address that no check dereferences
no_device = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="calls that are not refused would be launched")


def _at(n, first=0, off=0):
    return None if n is None else (ctypes.c_void_p * max(n, 0))(*[GOOD + 4096 * (first + i) + off for i in range(n)])


def _list(places):
    return None if places is None else (ctypes.c_void_p * len(places))(*[GOOD + 4096 * i for i in places])


BAD, NO, DONE = sg.SG_ERR_INVALID_ARG, sg.SG_ERR_UNSUPPORTED, sg.SG_ERR_HIP   # (what passes the checks ends with the missing device's error)


# ------------------------------------------------------------------------------------------------ rotary positions
def _rotary(**fields):
    p = sg.make_rotary_problem((2, 3, 4), 4, 64, "bf16", (16, 24, 24), kv_heads=2)
    for name, value in fields.items():
        setattr(p, name, value)
    return p


@pytest.mark.parametrize("fields, status", [
    ({}, sg.SG_OK), ({"T": 0}, BAD), ({"H": -1}, BAD), ({"W": 0}, BAD), ({"heads": 0}, BAD), ({"kv_heads": -1}, BAD), ({"head_dim": 0}, BAD), ({"head_dim": 60}, BAD),
    ({"dtype": 2}, BAD), ({"dtype": 3}, BAD), ({"layout": 2}, BAD), ({"layout": -1}, BAD), ({"axis_t": 15}, BAD), ({"axis_t": -2, "axis_y": 40}, BAD),
    ({"axis_t": 18}, BAD), ({"axis_t": 0, "axis_y": 0, "axis_x": 0}, BAD), ({"axis_t": 0, "axis_y": 0, "axis_x": 2}, sg.SG_OK),
    ({"layout": 1}, sg.SG_OK), ({"layout": 1, "axis_t": 14}, NO), ({"axis_t": 14}, sg.SG_OK), ({"canvas_h": -1}, BAD),
    ({"position_axes": 2}, BAD), ({"position_axes": 3}, sg.SG_OK), ({"eps": -1.0}, BAD), ({"eps": float("nan")}, BAD), ({"eps": float("inf")}, BAD), ({"eps": 0.0}, sg.SG_OK),
    ({"q_stride_token": 60}, BAD), ({"q_stride_token": 56}, BAD), ({"q_stride_head": 0}, BAD), ({"q_stride_head": 8}, sg.SG_OK),
    ({"q_out_stride_head": 8}, BAD), ({"q_out_stride_head": 64}, BAD), ({"q_out_stride_head": 64, "q_out_stride_token": 256}, sg.SG_OK),
    ({"k_out_stride_head": 64}, BAD), ({"k_out_stride_head": 64, "kv_heads": 1}, sg.SG_OK), ({"k_stride_token": 1 << 40}, BAD),
    ({"T": 1 << 12, "H": 1 << 12, "W": 1}, NO), ({"T": 1 << 30, "H": 1 << 30, "W": 1 << 30}, NO),
    ({"head_dim": 520, "q_stride_token": 520, "q_out_stride_token": 520, "k_stride_token": 520, "k_out_stride_token": 520, "q_out_stride_head": 520 * 24,
      "k_out_stride_head": 520 * 24}, NO),
])
def test_rotary_problem_is_checked(fields, status):
    assert sg.sg_rotary_validate(_rotary(**fields)) == status


def _turn(p=None, n=2, **kw):
    a = dict(q=_at(n), k=_at(n, 10), freq=GOOD, origin=(ctypes.c_int32 * (3 * max(n, 1)))(), positions=None, wq=None, wk=None, run=None, qo=_at(n, 20), ko=_at(n, 30))
    a.update(kw)
    p = p or _rotary()
    return sg.load_library().sg_tile_rotary(ctypes.byref(p), n, a["q"], a["k"], a["freq"], a["origin"], a["positions"], a["wq"], a["wk"], a["run"], a["qo"],
                                            a["ko"], None)


def test_rotary_calls_are_refused():
    origin = (ctypes.c_int32 * 6)()
    far = (ctypes.c_int32 * 6)(0, 0, 0, 0, 2 ** 31 - 1, 0)
    assert _turn(n=0) == sg.SG_OK and _turn(n=-1, q=None) == BAD
    for kw in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(freq=None), dict(freq=GOOD + 4), dict(origin=None), dict(positions=_at(2, 40)),
               dict(q=_at(2, 0, 8)), dict(qo=_at(2, 20, 4)), dict(wq=GOOD + 8), dict(wk=GOOD + 2), dict(origin=None, positions=_at(2, 40, 2)), dict(origin=far),
               dict(qo=_list([20, 20])), dict(qo=_list([1, 0])), dict(qo=_list([10, 21])), dict(ko=_list([0, 31])), dict(ko=_list([20, 31])),
               dict(p=_rotary(q_out_stride_token=72, q_out_stride_head=72 * 24), qo=_at(2))):
        assert _turn(**kw) == BAD, kw
    assert _turn(n=257, q=_at(257), k=None, ko=None, qo=_at(257, 300)) == NO
    assert _turn(p=_rotary(kv_heads=0)) == BAD
    assert origin[0] == 0


@no_device
def test_rotary_calls_that_are_not():
    for kw in ({}, dict(qo=_at(2)), dict(qo=_at(2), ko=_at(2, 10)), dict(k=None, ko=None), dict(origin=None, positions=_at(2, 40, 4)), dict(wq=GOOD, wk=GOOD + 16),
               dict(p=_rotary(canvas_h=9), origin=(ctypes.c_int32 * 6)(0, 0, 0, 0, 2 ** 31 - 1, 0)), dict(p=_rotary(kv_heads=0), k=None, ko=None), dict(q=_list([0, 0]))):
        assert _turn(**kw) == DONE, kw


def test_rotary_frequencies():
    p = _rotary(axis_t=2, axis_y=24, axis_x=16)
    for scaling, factor in (("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("ramp", 2.0)):
        got = sg.sg_rotary_frequencies(p, base=500.0, scaling=scaling, factor=factor, length=300.0, slow=1.0, fast=16.0, device="cpu")
        want = []
        for n in (2, 24, 16):
            base = 500.0 * factor ** (n / (n - 2)) if scaling == "ntk" and n > 2 else 500.0
            for i in range(n // 2):
                f = math.exp(-2 * i / n * math.log(base))
                turns = 300.0 * f / (2 * math.pi)
                if scaling == "linear":
                    f = f / 4.0
                if scaling == "ramp" and turns < 16:
                    f = f / 2 if turns <= 1 else f * ((turns - 1) / 15) + f / 2 * (1 - (turns - 1) / 15)
                want.append(f)
        assert got.dtype == torch.float64 and got.shape == (21,)
        # a power and a logarithm in fp64, each argument below 7
        assert torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=64 * 2.0 ** -53, atol=0)
    last = sg.sg_rotary_frequencies(p, scaling="ntk", factor=8.0, device="cpu")[12] / sg.sg_rotary_frequencies(p, device="cpu")[12]
    assert abs(float(last) - 1 / 8) < 1e-12   # the last pair is stretched by the whole factor


@pytest.mark.parametrize("kw", [dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.0), dict(scaling="ntk", factor=-1.0),
                                dict(scaling="ramp", factor=2.0, length=0.0), dict(scaling="ramp", factor=2.0, length=9.0, slow=3.0, fast=3.0),
                                dict(scaling="ramp", factor=2.0, length=9.0, slow=-1.0), dict(scaling="ramp", factor=float("inf"), length=9.0)])
def test_frequencies_are_refused(kw):
    with pytest.raises(sg.SgError):
        sg.sg_rotary_frequencies(_rotary(), device="cpu", **kw)


def test_frequencies_of_another_scaling_or_problem_are_refused():
    lib, out = sg.load_library(), (ctypes.c_double * 64)()
    call = lambda p, scaling: lib.sg_rotary_frequencies(p, 1e4, scaling, 1.0, 1.0, 1.0, 2.0, out)   # noqa: E731
    assert call(ctypes.byref(_rotary()), 4) == BAD and call(ctypes.byref(_rotary()), -1) == BAD and call(None, 0) == BAD
    assert call(ctypes.byref(_rotary(axis_t=80)), 0) == BAD and lib.sg_rotary_frequencies(ctypes.byref(_rotary()), 1e4, 0, 1.0, 1.0, 1.0, 2.0, None) == BAD


def test_binding_refuses_other_tensors():
    p = _rotary()
    t = torch.zeros(8)
    with pytest.raises(TypeError):
        sg.sg_tile_rotary(p, [t], [t], torch.zeros(32), origin=[(0, 0, 0)])
    with pytest.raises(ValueError):
        sg.sg_tile_rotary(p, [t], [t], torch.zeros(32, dtype=torch.float64), origin=[(0, 0, 0), (0, 0, 0)])
    with pytest.raises(TypeError):
        sg.sg_tile_rotary(p, [t], [t], torch.zeros(32, dtype=torch.float64), positions=[torch.zeros(24, dtype=torch.int64)])
    with pytest.raises(TypeError):
        sg.sg_tile_int8_linear(sg.make_int8_linear_problem(1, 16, 8, "f32"), [t.to(torch.uint8)], [t], t.to(torch.int8), t, [t])
    with pytest.raises(TypeError):
        sg.sg_tile_int8_linear(sg.make_int8_linear_problem(1, 16, 8, "f32"), [t.to(torch.int8)], [t.double()], t.to(torch.int8), t, [t])


# ------------------------------------------------------------------------------------------------ gated norm
def _norm(n=2, fields=None, **kw):
    p = sg.make_gated_norm_problem(5, 256, "bf16", post_norm="rms")
    a = dict(x=range(n), residual=range(100, 100 + n), gate=range(200, 200 + n), scale=range(300, 300 + n), shift=range(400, 400 + n), total=range(500, 500 + n),
             out=range(600, 600 + n), out_scale=None, weight=None, post_weight=None)
    a.update(kw)
    for name, value in (fields or {}).items():
        setattr(p, name, value)
    arr = lambda v: v if isinstance(v, ctypes.Array) else _list(v)   # noqa: E731
    return sg.load_library().sg_tile_gated_norm(ctypes.byref(p), n, arr(a["x"]), arr(a["residual"]), arr(a["gate"]), a["post_weight"], a["weight"], arr(a["scale"]),
                                                arr(a["shift"]), None, arr(a["total"]), arr(a["out"]), arr(a["out_scale"]), None)


@pytest.mark.parametrize("kw, status", [
    (dict(fields={"rows": -1}), BAD), (dict(fields={"rows": 0}), sg.SG_OK), (dict(n=0), sg.SG_OK), (dict(fields={"channels": 0}), BAD),
    (dict(fields={"channels": 100}), BAD), (dict(fields={"dtype": 2}), BAD), (dict(fields={"out_dtype": 0}), BAD), (dict(fields={"out_dtype": 4}), BAD),
    (dict(fields={"scale_group": 128}), BAD), (dict(fields={"out_dtype": 3, "scale_group": 100}, out_scale=range(700, 702)), BAD),
    (dict(fields={"out_dtype": 3, "scale_group": 64}, out_scale=range(700, 702)), NO), (dict(fields={"out_dtype": 3}), BAD), (dict(out_scale=range(700, 702)), BAD),
    (dict(fields={"norm": 0}), BAD), (dict(fields={"norm": 3}), BAD), (dict(fields={"post_norm": 3}), BAD), (dict(fields={"mod_dtype": 2}), BAD),
    (dict(fields={"dtype": 0, "out_dtype": 0, "mod_dtype": 1}), BAD), (dict(fields={"mod_rows": -1}), BAD), (dict(fields={"mod_rows": 2, "mod_stride": 248}), BAD),
    (dict(fields={"mod_rows": 2, "mod_stride": 260}), BAD), (dict(fields={"residual_scale": float("nan")}), BAD), (dict(fields={"eps": -1e-6}), BAD),
    (dict(fields={"post_eps": float("inf")}), BAD), (dict(fields={"x_stride": 248}), BAD), (dict(fields={"out_stride": 257}), BAD), (dict(fields={"sum_stride": 0}), BAD),
    (dict(fields={"residual_stride": 0}), BAD), (dict(fields={"post_norm": 0}, post_weight=GOOD), BAD), (dict(weight=GOOD + 8), BAD), (dict(x=None), BAD), (dict(out=None), BAD),
    (dict(gate=_at(2, 200, 8)), BAD), (dict(scale=_at(2, 300, 4)), BAD), (dict(shift=(ctypes.c_void_p * 2)()), BAD),
    (dict(out=[0, 601]), BAD), (dict(out=[100, 601]), BAD), (dict(out=[600, 600]), BAD), (dict(out=[500, 601]), BAD), (dict(out=[201, 601]), BAD), (dict(out=[400, 601]), BAD),
    (dict(total=[500, 500]), BAD), (dict(total=[1, 500]), BAD), (dict(total=[300, 500]), BAD), (dict(total=[0, 1], fields={"sum_stride": 512}), BAD),
    (dict(total=[100, 101], fields={"residual_stride": 512}), BAD), (dict(fields={"channels": 32776, "x_stride": 32776, "residual_stride": 32776, "sum_stride": 32776,
                                                                                 "out_stride": 32776}), NO),
    (dict(n=257), NO),
])
def test_gated_norms_are_refused(kw, status):
    assert _norm(**kw) == status


@no_device
@pytest.mark.parametrize("kw", [
    {}, dict(total=[0, 1]), dict(total=[100, 101]), dict(total=None), dict(residual=None, fields={"residual_scale": float("nan"), "residual_stride": 0}), dict(gate=None, scale=None),
    dict(x=[0, 0]), dict(gate=[200, 200], scale=[200, 200]), dict(fields={"mod_rows": 9, "mod_stride": 0}), dict(fields={"out_dtype": 3}, out_scale=range(700, 702)),
    dict(fields={"out_dtype": 2, "scale_group": 128}, out_scale=_at(2, 700, 4)), dict(fields={"mod_dtype": 0}), dict(weight=GOOD, post_weight=GOOD)])
def test_gated_norms_that_are_not(kw):
    assert _norm(**kw) == DONE


# ------------------------------------------------------------------------------------------------ linear layer
@pytest.mark.parametrize("fields, status", [
    ({}, sg.SG_OK), ({"rows": 0}, sg.SG_OK), ({"rows": -1}, BAD), ({"channels": 0}, BAD), ({"channels": 72}, BAD), ({"outputs": 0}, BAD), ({"outputs": 12}, BAD),
    ({"dtype": 2}, BAD), ({"dtype": 3}, BAD), ({"activation": 2}, BAD), ({"activation": -1}, BAD), ({"x_stride": 48}, BAD), ({"x_stride": 72}, BAD), ({"w_stride": 0}, BAD),
    ({"out_stride": 32}, BAD), ({"out_stride": 44}, BAD), ({"x_stride": 1 << 40}, BAD), ({"channels": 131072, "x_stride": 131072, "w_stride": 131072}, NO),
    ({"channels": 131056, "x_stride": 131056, "w_stride": 131056}, sg.SG_OK), ({"outputs": 1 << 26, "out_stride": 1 << 26}, sg.SG_OK),
    ({"outputs": (1 << 26) + 8, "out_stride": (1 << 26) + 8}, NO)])
def test_linear_problem_is_checked(fields, status):
    p = sg.make_int8_linear_problem(6, 64, 40, "bf16")
    for name, value in fields.items():
        setattr(p, name, value)
    assert sg.sg_int8_linear_validate(p) == status


def _linear(n=2, fields=None, **kw):
    p = sg.make_int8_linear_problem(6, 64, 40, "bf16")
    for name, value in (fields or {}).items():
        setattr(p, name, value)
    a = dict(x=_at(n), x_scale=_at(n, 300), w=GOOD, w_scale=GOOD, bias=GOOD, out=_at(n, 600))
    a.update(kw)
    return sg.load_library().sg_tile_int8_linear(ctypes.byref(p), n, a["x"], a["x_scale"], a["w"], a["w_scale"], a["bias"], None, a["out"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(n=0), sg.SG_OK), (dict(fields={"rows": 0}), sg.SG_OK), (dict(n=-1, x=None), BAD), (dict(n=257), NO), (dict(x=None), BAD), (dict(x_scale=None), BAD), (dict(out=None), BAD),
    (dict(w=None), BAD), (dict(w_scale=None), BAD), (dict(w=GOOD + 8), BAD), (dict(w_scale=GOOD + 4), BAD), (dict(bias=GOOD + 2), BAD), (dict(x=_at(2, 0, 8)), BAD),
    (dict(x_scale=_at(2, 300, 2)), BAD), (dict(out=_at(2, 600, 4)), BAD), (dict(out=_at(2)), BAD), (dict(out=_list([600, 600])), BAD),
    (dict(fields={"rows": 1 << 30}), NO), (dict(fields={"rows": 1 << 20, "outputs": 1 << 19, "out_stride": 1 << 19}), NO),
    (dict(fields={"outputs": (1 << 26) + 8, "out_stride": (1 << 26) + 8}), NO), (dict(fields={"rows": 257, "outputs": 1 << 26, "out_stride": 1 << 26}, n=64), NO)])
def test_linear_calls_are_refused(kw, status):
    assert _linear(**kw) == status


@no_device
@pytest.mark.parametrize("kw", [{}, dict(bias=None), dict(x=_list([0, 0])), dict(x_scale=_at(2, 300, 4)), dict(fields={"rows": 1 << 20, "outputs": 1 << 16, "out_stride": 1 << 16}),
                                dict(fields={"rows": (1 << 29) - 1}), dict(n=1, fields={"rows": 1, "outputs": 1 << 26, "out_stride": 1 << 26}),
                                dict(n=1, fields={"rows": 64, "outputs": 1 << 26, "out_stride": 1 << 26})])
def test_linear_calls_that_are_not(kw):
    assert _linear(**kw) == DONE
