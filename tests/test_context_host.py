"""Argument checks of the context attentions and the residual norm, on the host: a call that cannot be made is refused before anything
is launched (no GPU is touched here)."""
import ctypes

import pytest

import paper_2508_17756_amd as sg

GOOD = 0x10000   # an aligned address that no check dereferences


def _array(n, value=GOOD):
    return (ctypes.c_void_p * n)(*[value + 4096 * i for i in range(n)])


def _problem(**fields):
    p = sg.make_context_problem(12, 20, 4, 64, "bf16", kv_heads=2, own_tokens=12)
    for name, value in fields.items():
        setattr(p, name, value)
    return p


@pytest.mark.parametrize("fields, status", [
    ({}, sg.SG_OK),
    ({"ctx_tokens": 0}, sg.SG_OK), ({"own_tokens": 0}, sg.SG_OK), ({"tokens": 1}, sg.SG_OK), ({"kv_heads": 4}, sg.SG_OK),
    ({"heads": 0}, sg.SG_ERR_INVALID_ARG), ({"kv_heads": 0}, sg.SG_ERR_INVALID_ARG), ({"kv_heads": 3}, sg.SG_ERR_INVALID_ARG),
    ({"kv_heads": 8}, sg.SG_ERR_INVALID_ARG), ({"tokens": 0}, sg.SG_ERR_INVALID_ARG), ({"ctx_tokens": -1}, sg.SG_ERR_INVALID_ARG),
    ({"own_tokens": -1}, sg.SG_ERR_INVALID_ARG), ({"head_dim": 0}, sg.SG_ERR_INVALID_ARG),
    ({"dtype": 2}, sg.SG_ERR_INVALID_ARG), ({"dtype": -1}, sg.SG_ERR_INVALID_ARG),
    ({"scale": 0.0}, sg.SG_ERR_INVALID_ARG), ({"scale": -1.0}, sg.SG_ERR_INVALID_ARG), ({"scale": float("nan")}, sg.SG_ERR_INVALID_ARG),
    ({"scale": float("inf")}, sg.SG_ERR_INVALID_ARG),
    ({"q_stride_token": 63}, sg.SG_ERR_INVALID_ARG), ({"q_stride_token": 68}, sg.SG_ERR_INVALID_ARG),
    ({"ctx_stride_head": 0}, sg.SG_ERR_INVALID_ARG), ({"ctx_stride_head": -64}, sg.SG_ERR_INVALID_ARG),
    ({"own_stride_token": 56}, sg.SG_ERR_INVALID_ARG), ({"own_stride_token": 0, "own_tokens": 0}, sg.SG_OK),
    ({"ctx_stride_token": 0, "ctx_tokens": 0}, sg.SG_OK),
    ({"out_stride_head": 8}, sg.SG_ERR_INVALID_ARG), ({"out_stride_head": 64}, sg.SG_ERR_INVALID_ARG),   # heads would overlap
    ({"out_stride_head": 64, "out_stride_token": 256}, sg.SG_OK),                                         # heads inside a token
    ({"out_stride_head": 64, "tokens": 1}, sg.SG_OK),
    ({"out_stride_head": 8, "heads": 1, "kv_heads": 1}, sg.SG_OK),
    ({"head_dim": 128, "q_stride_token": 128, "ctx_stride_token": 128, "own_stride_token": 128, "out_stride_token": 128,
      "out_stride_head": 12 * 128}, sg.SG_OK),
    ({"head_dim": 32}, sg.SG_ERR_UNSUPPORTED), ({"ctx_stride_token": 1 << 22}, sg.SG_ERR_UNSUPPORTED),
    ({"heads": 65536, "kv_heads": 65536, "tokens": 1}, sg.SG_ERR_UNSUPPORTED), ({"heads": 65536, "kv_heads": 32768, "tokens": 1}, sg.SG_OK),
    ({"own_stride_token": 1 << 22}, sg.SG_ERR_UNSUPPORTED), ({"tokens": 1 << 23, "out_stride_head": 64 << 23}, sg.SG_ERR_UNSUPPORTED),
])
def test_context_problem_is_checked(fields, status):
    p = _problem(**fields)
    assert sg.sg_context_validate(p) == status
    n = ctypes.c_size_t(7)
    assert sg.load_library().sg_context_workspace_bytes(ctypes.byref(p), 3, ctypes.byref(n)) == status
    assert (n.value == 7) == (status != sg.SG_OK)


def test_workspace_bytes_refuses_and_grows():
    lib, p, n = sg.load_library(), _problem(), ctypes.c_size_t(7)
    assert lib.sg_context_workspace_bytes(ctypes.byref(p), -1, ctypes.byref(n)) == sg.SG_ERR_INVALID_ARG
    assert lib.sg_context_workspace_bytes(ctypes.byref(p), 3, None) == sg.SG_ERR_INVALID_ARG
    assert lib.sg_context_workspace_bytes(ctypes.byref(p), 257, ctypes.byref(n)) == sg.SG_ERR_UNSUPPORTED
    assert lib.sg_context_workspace_bytes(None, 3, ctypes.byref(n)) == sg.SG_ERR_INVALID_ARG and n.value == 7
    assert sg.sg_context_workspace_bytes(p, 0) == 0
    long = sg.make_context_problem(1, 30000, 8, 128, "bf16", own_tokens=200)
    assert sg.sg_context_workspace_bytes(long, 4) > 0 and sg.sg_context_workspace_bytes(long, 4) % 256 == 0
    # a call of more tiles than a launch takes needs what its largest launch does
    assert sg.sg_context_workspace_bytes(long, 130) >= sg.sg_context_workspace_bytes(long, 64)


def _cross(p, n, q, k, v, out, ws=None, bytes_=0):
    return sg.load_library().sg_tile_cross_attention(ctypes.byref(p) if p is not None else None, n, q, k, v, None, None, None, out, ws, bytes_, None)


def _prefix(p, n, q, k, v, pk, pv, out, ws=None, bytes_=0):
    return sg.load_library().sg_tile_prefix_attention(ctypes.byref(p) if p is not None else None, n, q, k, v, pk, pv, None, None, None, out, ws,
                                                      bytes_, None)


def test_attention_calls_are_refused():
    bad, none, p = sg.SG_ERR_INVALID_ARG, None, _problem()
    a, odd, hole = _array(3), _array(3, GOOD + 8), (ctypes.c_void_p * 3)(GOOD, None, GOOD)
    assert _cross(None, 3, a, a, a, a) == bad and _cross(_problem(heads=0), 3, a, a, a, a) == bad
    assert _cross(p, -1, a, a, a, a) == bad and _cross(p, 257, a, a, a, a) == sg.SG_ERR_UNSUPPORTED
    assert _cross(p, 0, none, none, none, none) == sg.SG_OK
    for wrong in (none, odd, hole):
        assert _cross(p, 3, wrong, a, a, a) == bad and _cross(p, 3, a, wrong, a, a) == bad
        assert _cross(p, 3, a, a, wrong, a) == bad and _cross(p, 3, a, a, a, wrong) == bad
        assert _prefix(p, 3, wrong, a, a, GOOD, GOOD, a) == bad and _prefix(p, 3, a, wrong, a, GOOD, GOOD, a) == bad
        assert _prefix(p, 3, a, a, wrong, GOOD, GOOD, a) == bad and _prefix(p, 3, a, a, a, GOOD, GOOD, wrong) == bad
    for wrong in (none, GOOD + 8):
        assert _prefix(p, 3, a, a, a, wrong, GOOD, a) == bad and _prefix(p, 3, a, a, a, GOOD, wrong, a) == bad
    assert _prefix(None, 3, a, a, a, GOOD, GOOD, a) == bad and _prefix(p, -1, a, a, a, GOOD, GOOD, a) == bad
    assert _prefix(p, 0, none, none, none, none, none, none) == sg.SG_OK


def test_a_call_that_joins_shares_needs_its_workspace():
    p = sg.make_context_problem(1, 30000, 8, 128, "bf16", own_tokens=200)
    need, a = sg.sg_context_workspace_bytes(p, 2), _array(2)
    assert need > 0
    for ws, size in ((None, need), (GOOD + 16, need), (GOOD, 255), (GOOD, 0)):
        assert _prefix(p, 2, a, a, a, GOOD, GOOD, a, ws, size) == sg.SG_ERR_WORKSPACE
        assert _cross(p, 2, a, a, a, a, ws, size) == sg.SG_ERR_WORKSPACE
    assert _prefix(p, 2, a, a, a, GOOD, GOOD, a, GOOD, need - 256) in (sg.SG_ERR_WORKSPACE,) or \
        _cross(p, 2, a, a, a, a, GOOD, need - 256) == sg.SG_ERR_WORKSPACE


def _norm(p, n=2, x=True, residual=None, weight=None, total=None, out=True, scale=None):
    arr = lambda v: _array(n) if v is True else v   # noqa: E731
    return sg.load_library().sg_tile_residual_norm(ctypes.byref(p) if p is not None else None, n, arr(x), arr(residual), weight, None,
                                                   arr(total), arr(out), arr(scale), None)


@pytest.mark.parametrize("fields, status", [
    ({"rows": -1}, sg.SG_ERR_INVALID_ARG), ({"channels": 0}, sg.SG_ERR_INVALID_ARG), ({"channels": 100}, sg.SG_ERR_INVALID_ARG),
    ({"dtype": 2}, sg.SG_ERR_INVALID_ARG), ({"dtype": 5}, sg.SG_ERR_INVALID_ARG), ({"out_dtype": 0}, sg.SG_ERR_INVALID_ARG),
    ({"out_dtype": 3}, sg.SG_ERR_INVALID_ARG), ({"eps": -1.0}, sg.SG_ERR_INVALID_ARG), ({"eps": float("nan")}, sg.SG_ERR_INVALID_ARG),
    ({"x_stride": 248}, sg.SG_ERR_INVALID_ARG), ({"x_stride": 260}, sg.SG_ERR_INVALID_ARG), ({"out_stride": 0}, sg.SG_ERR_INVALID_ARG),
    ({"residual_stride": 8}, sg.SG_ERR_INVALID_ARG), ({"sum_stride": 8}, sg.SG_ERR_INVALID_ARG),
    ({"scale_group": 128}, sg.SG_ERR_INVALID_ARG),   # not an output in 8 bits
    ({"channels": 32776, "x_stride": 32776, "residual_stride": 32776, "sum_stride": 32776, "out_stride": 32776}, sg.SG_ERR_UNSUPPORTED),
])
def test_norm_problem_is_checked(fields, status):
    p = sg.make_norm_problem(5, 256, "bf16")
    for name, value in fields.items():
        setattr(p, name, value)
    assert _norm(p, residual=True, total=True) == status


def test_norm_calls_are_refused():
    bad = sg.SG_ERR_INVALID_ARG
    p, p8 = sg.make_norm_problem(5, 256, "bf16"), sg.make_norm_problem(5, 256, "bf16", out_dtype="e4m3", scale_group=128)
    odd, hole = _array(2, GOOD + 8), (ctypes.c_void_p * 2)(GOOD, None)
    assert _norm(None) == bad and _norm(p, n=-1, x=None, out=None) == bad
    assert _norm(p, n=0, x=None, out=None) == sg.SG_OK and _norm(p, n=257) == sg.SG_ERR_UNSUPPORTED
    empty = sg.make_norm_problem(0, 256, "bf16")
    assert _norm(empty, x=None, out=None) == sg.SG_OK
    for wrong in (None, odd, hole):
        assert _norm(p, x=wrong) == bad and _norm(p, out=wrong) == bad
    for wrong in (odd, hole):
        assert _norm(p, residual=wrong) == bad and _norm(p, total=wrong) == bad
    assert _norm(p, weight=GOOD + 8) == bad
    assert _norm(p, scale=True) == bad            # no output in 8 bits
    assert _norm(p8) == bad                       # scales missing
    assert _norm(p8, scale=hole) == bad and _norm(p8, scale=_array(2, GOOD + 2)) == bad
    for group, status in ((96, bad), (-128, bad), (64, sg.SG_ERR_UNSUPPORTED), (256, sg.SG_ERR_UNSUPPORTED)):
        p8.scale_group = group
        assert _norm(p8, scale=True) == status, group


class _Host:
    """A tensor's stand-in for the binding."""

    def data_ptr(self):
        return GOOD


def test_lists_of_unequal_length_are_refused():
    """The library reads one pointer per tile from each list."""
    p, two, one = _problem(), [_Host()] * 2, [_Host()]
    for k, v, out in ((one, two, two), (two, one, two), (two, two, one), (two, two, two + one)):
        with pytest.raises(ValueError):
            sg.sg_tile_cross_attention(p, two, k, v, out)
        with pytest.raises(ValueError):
            sg.sg_tile_prefix_attention(p, two, k, v, _Host(), _Host(), out)
    n = sg.make_norm_problem(5, 256, "bf16")
    for lists in ({"out": one}, {"residual": one}, {"sum_out": one}, {"out_scale": one}):
        with pytest.raises(ValueError):
            sg.sg_tile_residual_norm(n, two, None, **{"out": two, **lists})
