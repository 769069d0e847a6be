"""The residual norm over the whole range of its types: squares whose sum leaves the fp32 range on either side, scales of rows with a NaN."""
import pytest
import torch

import paper_2508_17756_amd as sg
from context_util import TORCH, U8, U16, U32, norm64
from test_gpu_residual_norm import _call, _check

pytestmark = pytest.mark.gpu

CHANNELS = [64, 128, 1024, 5120, 32768]   # 8 rows to a wavefront, 4, half a row to a lane's vectors, 4 wavefronts, 16 wavefronts


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("gain", [2.0 ** 55, 2.0 ** 59, 2.0 ** 62, 2.0 ** 90, 2.0 ** 120])
def test_large_rows(dtype, channels, gain):
    """Values of up to about 5 x gain, the sum of whose squares passes 2^128 (1,024 channels of 2^59 do)."""
    _check(*_call(2, 5, channels, dtype, gain=gain, seed=channels), dtype)
    _check(*_call(1, 5, channels, dtype, out_dtype="e4m3", gain=gain, pad=8, residual=False, seed=channels + 1), dtype)
    if channels % 128 == 0:
        _check(*_call(1, 5, channels, dtype, out_dtype="e4m3", group=128, gain=gain, seed=channels + 2), dtype, group=128)


def _rows(channels, dtype, magnitudes, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((len(magnitudes), channels), generator=g, dtype=torch.float64)
    return (x * torch.tensor(magnitudes, dtype=torch.float64)[:, None]).to(TORCH[dtype]).cuda()


def _tolerance(y, channels, dtype):
    """The sum of squares is off by at most (channels / 2 + 8) 2^-24 of itself, the root, its reciprocal and the products by 8 roundings, then the
    store (as in test_gpu_residual_norm; there is no residual, so nothing cancels)."""
    return ((channels / 4 + 16) * U32 + (U16 if dtype == "bf16" else U32)) * 1.01 * y.abs() + 1e-30


MIXED = [1.0, 2.0 ** 100, 2.0 ** -30, 2.0 ** 64, 2.0 ** 20, 2.0 ** 60, 2.0 ** 121, 0.5]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("eps", [1e-6, 0.0, 1e30])
def test_rows_of_every_size_beside_one_another(dtype, channels, eps):
    """Rows that need another scale share wavefronts and workgroups with rows that do not; the sum is stored as it is."""
    x, r = _rows(channels, dtype, MIXED * 3, 1), _rows(channels, dtype, MIXED * 3, 2)
    p = sg.make_norm_problem(24, channels, dtype, eps=eps)
    s, y = torch.empty_like(x), torch.empty_like(x)
    sg.sg_tile_residual_norm(p, [x], None, [y], sum_out=[s], residual=[r])
    torch.cuda.synchronize()
    assert torch.equal(s.cpu(), (x.cpu().float() + r.cpu().float()).to(x.dtype))
    total, want = norm64(x.cpu(), r.cpu(), None, p.eps)
    mag = x.cpu().double().abs() + r.cpu().double().abs()
    tol = _tolerance(want, channels, dtype) + 2 * U32 * (want / total.where(total != 0, torch.ones_like(total))).abs() * mag
    assert bool(((y.cpu().double() - want).abs() <= tol).all())


# 2^-140 is below the smallest normal number of either type, which has 2^-149 (bf16: 2^-133) for its smallest
@pytest.mark.parametrize("dtype, least", [("f32", -140), ("bf16", -126)])
@pytest.mark.parametrize("channels", CHANNELS)
def test_small_rows_without_eps(dtype, least, channels):
    sizes = [2.0 ** -40, 2.0 ** -49, 2.0 ** -51, 2.0 ** -63, 2.0 ** -70, 1.0, 2.0 ** -76, 2.0 ** -90, 2.0 ** -110, 2.0 ** least, 2.0 ** 100]
    x = _rows(channels, dtype, sizes, 3)
    for eps in (0.0, 1e-42, 2.0 ** -110):
        p = sg.make_norm_problem(len(sizes), channels, dtype, eps=eps)
        y = torch.empty_like(x)
        sg.sg_tile_residual_norm(p, [x], None, [y])
        p8 = sg.make_norm_problem(len(sizes), channels, dtype, out_dtype="e4m3", eps=eps)
        y8, scale = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((len(sizes), 1), device="cuda")
        sg.sg_tile_residual_norm(p8, [x], None, [y8], out_scale=[scale])
        torch.cuda.synchronize()
        _, want = norm64(x.cpu(), None, None, p.eps)
        assert bool(((y.cpu().double() - want).abs() <= _tolerance(want, channels, dtype)).all()), eps
        sc = scale.cpu().double()
        tol = _tolerance(want, channels, "f32") * (1 + U8) + (U8 + 8 * U32) * want.abs() + 2.0 ** -10 * sc + 2.0 ** -100
        assert bool(((y8.cpu().float().double() * sc - want).abs() <= tol).all()), eps


def test_a_row_of_zeros_without_eps_is_nan_and_with_any_eps_zeros():
    for channels in CHANNELS:
        x = torch.zeros((3, channels), device="cuda")
        x[1] = 1.0
        for eps in (0.0, 1e-42, 1e-6):
            y = torch.empty_like(x)
            sg.sg_tile_residual_norm(sg.make_norm_problem(3, channels, "f32", eps=eps), [x], None, [y])
            torch.cuda.synchronize()
            assert bool(torch.isnan(y[[0, 2]]).all()) if eps == 0 else bool((y[[0, 2]] == 0).all())
            assert float((y[1] - 1).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", CHANNELS[1:])
@pytest.mark.parametrize("group", [0, 128])
def test_scales_of_rows_with_a_nan(dtype, channels, group):
    """Codes and scales both: what leaves out blocks whose scale is 0 must not lose a NaN.  A NaN in the weight is one of its block."""
    x = _rows(channels, dtype, [1.0] * 9, 4)
    x[2, channels // 2] = float("nan")
    x[5, channels - 1] = float("nan")
    x[7] = 0
    w = torch.ones(channels, device="cuda").to(x.dtype)
    p = sg.make_norm_problem(9, channels, dtype, out_dtype="e4m3", scale_group=group)
    y = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty((9, channels // group if group else 1), device="cuda")

    def call():
        sg.sg_tile_residual_norm(p, [x], w, [y], out_scale=[scale])
        torch.cuda.synchronize()
        return y.float().cpu(), scale.cpu()

    code, sc = call()
    for row in range(9):
        if row in (2, 5):
            assert bool(torch.isnan(code[row]).all()) and bool(torch.isnan(sc[row]).all())
        else:
            assert bool(torch.isfinite(code[row]).all()) and bool(torch.isfinite(sc[row]).all())
    assert float(sc[7].max()) == 0 and float(code[7].abs().max()) == 0
    w[3] = float("nan")
    code, sc = call()
    width = group or channels
    assert bool(torch.isnan(code[0, 3])) and bool(torch.isnan(sc[:, 0]).all())
    assert bool(torch.isfinite(sc[0, 1:]).all()) and bool(torch.isfinite(code[0, width:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", CHANNELS[1:])
def test_a_row_with_an_infinity(dtype, channels):
    """Infinity over infinity is NaN, numbers over infinity are 0; in 8 bits the block of the infinity is NaN."""
    x = _rows(channels, dtype, [1.0] * 5, 5)
    x[1, channels - 2] = -float("inf")
    for group in (None, 0, 128):
        p = sg.make_norm_problem(5, channels, dtype, out_dtype=None if group is None else "e4m3", scale_group=group or 0)
        y = torch.empty(x.shape, dtype=x.dtype if group is None else torch.float8_e4m3fn, device="cuda")
        scale = None if group is None else [torch.empty((5, channels // group if group else 1), device="cuda")]
        sg.sg_tile_residual_norm(p, [x], None, [y], out_scale=scale)
        torch.cuda.synchronize()
        got = y.float().cpu()
        want = torch.zeros(x.shape, dtype=torch.bool)
        if group is None:
            want[1, channels - 2] = True
        else:
            want[1, channels - (group or channels):] = True
            assert bool(torch.isnan(scale[0][1, -1])) and bool(torch.isfinite(scale[0][[0, 2, 3, 4]]).all())
        assert torch.equal(torch.isnan(got), want)
        assert bool((got[1][~want[1]] == 0).all())
