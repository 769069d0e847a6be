"""Layer norms of rows of one value, or nearly one: the deviations are zero, or a few steps of the values, however large those are, and count against eps."""
import pytest
import torch

import paper_2508_17756_amd as sg
from block_util import TORCH

pytestmark = pytest.mark.gpu

CHANNELS = [8, 64, 136, 256, 264, 512, 640, 1536, 5120, 8192, 20000, 32768]
# A sum of a row: a lane adds up to 32 terms in order (32 roundings), 6 exchanges between lanes, up to 15 additions of wavefronts.
SUM = 53 * 2.0 ** -24


def _norm(x, norm, post="none", eps=1e-6, out=None, group=0, shift=None):
    rows, channels = x.shape
    dtype = "f32" if x.dtype is torch.float32 else "bf16"
    p = sg.make_gated_norm_problem(rows, channels, dtype, out_dtype=out, scale_group=group, norm=norm, post_norm=post, eps=eps, post_eps=eps)
    kind = {None: x.dtype, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[out]
    y = torch.full((rows, channels), 1, dtype=torch.float32, device="cuda").to(kind)
    scale = torch.full((rows, channels // group if group else 1), -1.0, device="cuda") if out else None
    sg.sg_tile_gated_norm(p, [x], [y], out_scale=[scale] if out else None, shift=[shift] if shift is not None else None)
    torch.cuda.synchronize()
    return y, scale


def _values(dtype):
    """A value a row: every size from 1e-37 to the largest, both signs, mantissas of all kinds (their multiples round differently)."""
    g = torch.Generator().manual_seed(77)
    v = 10.0 ** (torch.rand(400, generator=g, dtype=torch.float64) * 75 - 37) * (1 - 2 * torch.randint(0, 2, (400,), generator=g))
    v = torch.cat([v, torch.tensor([0.0, 1.0, 3.0, -7.0, 1e4, 1e30, -1e35, 1e38, -3.3e38], dtype=torch.float64)])
    return v.float().to(TORCH[dtype]).cuda()


def _left(x):
    """What may be left of (v - mean) / sqrt(eps).  A mean is off by nothing or by a step of v at least, 2^-24 |v|; from |v| = 2^-50 on the square of that is no less than
    2^-148 and shows that the mean has to be taken again, between v and v.  Below, squares vanish: the mean is off by SUM |v|, a product and a difference
    by a rounding each."""
    v = x.double().abs()
    return torch.where(v < 2.0 ** -50, (SUM + 4 * 2.0 ** -24) * v, 0.0) / 1e-6 ** 0.5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("channels", CHANNELS)
def test_rows_of_one_value_are_zero(dtype, channels):
    """(v - mean) is 0, and 0 / sqrt(0 + eps) is 0."""
    x = _values(dtype)[:, None].expand(-1, channels).contiguous()
    left = _left(x)
    shift = torch.linspace(-2, 2, channels).to(TORCH[dtype]).cuda()[None]
    for kind, far in (("layer", 1.0), ("rms", 1e3)):   # (a norm behind it divides by sqrt(eps) once more)
        post = "layer" if kind == "rms" else "none"
        half = 2 * far * left   # (the rounding to the type)
        assert bool((_norm(x, kind, post=post)[0].double().abs() <= half).all())
        for out, top in (("e4m3", 448.0), ("int8", 127.0)):
            for group in (0, 128) if channels % 128 == 0 else (0,):
                y, scale = _norm(x, kind, post=post, out=out, group=group)
                each = scale.double().repeat_interleave(group or channels, dim=1)
                assert bool((y.double().abs() * each <= half).all()) and bool((each * top <= half).all()) and bool((y.float()[each == 0] == 0).all())
    assert bool((_norm(x, "layer", shift=shift)[0] == shift).all())


@pytest.mark.parametrize("channels", CHANNELS)
def test_without_an_eps_they_are_nan(channels):
    x = _values("f32")[:, None].expand(-1, channels).contiguous()
    y, _ = _norm(x, "layer", eps=0.0)
    assert bool(torch.isnan(y).all())


@pytest.mark.parametrize("channels", [64, 256, 264, 512])
@pytest.mark.parametrize("size", [1.0, 1e4, 1e8, 1e20, 1e33, 2e38])
def test_rows_of_nearly_one_value(channels, size):
    """Values m + k steps of m, k = 0 .. 4.  The mean lies between the least and the largest value, R apart, and what its rounding leaves is taken again with an error of
    SUM R; the variance, R^2 / channels at least, is off by SUM R^2 twice."""
    g = torch.Generator().manual_seed(int(channels + size % 97))
    rows = 60
    base = (size * (0.5 + torch.rand(rows, generator=g))).float().clamp(max=3.3e38)
    steps = torch.randint(0, 5, (rows, channels), generator=g)
    steps[::3] = 0
    steps[torch.arange(0, rows, 3), torch.randint(0, channels, (rows // 3,), generator=g)] = 3   # one that differs
    x = (base.view(torch.int32)[:, None] + steps.int()).view(torch.float32)
    got = _norm(x.cuda(), "layer")[0].cpu().double()
    d = x.double() - x.double().mean(dim=1, keepdim=True)
    spread = x.double().amax(dim=1, keepdim=True) - x.double().amin(dim=1, keepdim=True)
    var = d.square().mean(dim=1, keepdim=True)
    sigma = (var + float(torch.tensor(1e-6, dtype=torch.float32))).sqrt()
    ref = d / sigma
    tol = (2 * SUM * spread + 4 * 2.0 ** -24 * spread) / sigma + ref.abs() * (SUM * spread.square() / sigma.square() + 16 * 2.0 ** -24)
    off = (got - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("channels", [64, 640, 5120])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_nan_or_infinity_among_them_is_nan_throughout(channels, value):
    x = _values("f32")[:, None].expand(-1, channels).contiguous()
    clean = _norm(x, "layer")[0]
    x[5::7, channels // 3] = value
    y = _norm(x, "layer")[0]
    bad = torch.zeros(len(x), dtype=torch.bool, device="cuda")
    bad[5::7] = True
    assert bool(torch.isnan(y[bad]).all()) and torch.equal(y[~bad], clean[~bad])
