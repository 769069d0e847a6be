"""Norms with eps and of numbers at the ends of fp32's range, in front of what else a gated norm does and of rotary positions; a gated norm without gate and modulation in 8 bits
beside the residual norm: each result held against 64 bits or the other kernel."""
import pytest
import torch

import paper_2508_17756_amd as sg
import test_gpu_gated_norm
import test_gpu_rotary
from block_util import check_eight, gated64, same

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
SUM = 53 * U32   # 32 terms in a lane, 6 exchanges of lanes, 15 additions of wavefronts at most


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("channels", [64, 1024, 5120])
@pytest.mark.parametrize("gain", [1e37, 1e25, 1e-25, 1e-38])
def test_a_norm_of_far_numbers_in_front_of_gate_and_norm(norm, channels, gain):
    """x = gain * N(0, 1), no eps.  Behind the first norm everything is near 1."""
    c = test_gpu_gated_norm.Call(3, channels, "f32", post=norm, norm="rms", gain=gain, residual=False, eps=0.0).run()
    for i in range(2):
        x, gate = c.x[i].cpu().double(), c.gate[i][0].cpu().double() * c.post_weight.cpu().double()
        z = x - x.mean(dim=1, keepdim=True) if norm == "layer" else x
        z = z / z.square().mean(dim=1, keepdim=True).sqrt()
        # the norm's factor: half a sum's error, root, products; its mean SUM of the deviations.  Numbers below 2^-126 are multiples of 2^-149, so that a mean of x near
        # 2^-126 is off by 2^-24 of it and a difference by as much.
        err = (SUM + 10 * U32) * z.abs() + (2 * SUM + (4 * U32 if gain < 1e-30 else 0)) * (norm == "layer")
        s, es = z * gate, (err + 2 * U32 * z.abs()) * gate.abs()
        got = c.sum[i].cpu().double()
        assert bool(((got - s).abs() <= es + U32 * s.abs()).all()), float(((got - s).abs() / (es + U32 * s.abs())).max())
        sigma = s.square().mean(dim=1, keepdim=True).sqrt()
        w, b = 1 + c.scale[i][0].cpu().double(), c.shift[i][0].cpu().double()
        y = s / sigma * w + b
        ey = (es + (s / sigma).abs() * es.square().mean(dim=1, keepdim=True).sqrt()) / sigma * w.abs() + (SUM + 12 * U32) * (s / sigma * w).abs() + 2 * U32 * y.abs()
        got = c.out[i].cpu().double()
        assert bool(((got - y).abs() <= ey).all()), float(((got - y).abs() / ey).max())


@pytest.mark.parametrize("gain", [1e30, 1.0, 1e-3, 1e-6, 1e-30])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_heads_far_from_one_with_an_eps(gain, layout):
    """x * rsqrt(mean(x^2) + eps): eps counts nothing, something and everything."""
    eps = float(torch.tensor(1e-6, dtype=torch.float32))
    c = test_gpu_rotary.Call(dtype="f32", norm=True, gain=gain, heads=9, d=128, axes=(64, 32, 32), layout=layout, seed=4).run()
    for i in range(2):
        for key, xs, ys, weight in (("q", c.q, c.q_out, c.wq), ("k", c.k, c.k_out, c.wk)):
            x = c.view(xs[i], key).cpu().double()
            x = x / (x.square().mean(dim=-1, keepdim=True) + eps).sqrt() * weight.cpu().double()
            axis_of = torch.repeat_interleave(torch.arange(3), torch.tensor([n // 2 for n in c.axes]))
            w = (c.coords(i).double()[:, axis_of] * c.freq.cpu())[:, None, :]
            a, b = (x[..., :64], x[..., 64:]) if layout == "half" else (x[..., 0::2], x[..., 1::2])
            re, im = a * w.cos() - b * w.sin(), b * w.cos() + a * w.sin()
            y = torch.cat([re, im], dim=-1) if layout == "half" else torch.stack([re, im], dim=-1).flatten(-2)
            # 16 terms in a lane, 3 exchanges; root and two products; a sine within 2^-21; two products and their sum.  Numbers below 2^-126 in multiples of 2^-149.
            tol = (a.abs() + b.abs()) * (19 / 2 * U32 + 10 * U32 + 2.0 ** -21 + 3 * U32) + 2.0 ** -147
            tol = torch.cat([tol, tol], dim=-1) if layout == "half" else torch.stack([tol, tol], dim=-1).flatten(-2)
            off = (c.view(ys[i], key).cpu().double() - y).abs()
            assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", [128, 640, 5120])
def test_in_8_bits_it_is_the_residual_norm_without_gate_and_modulation(channels, dtype, group):
    c = test_gpu_gated_norm.Call(40, channels, dtype, gate=False, mod=False, weight=True, out="e4m3", group=group).run()
    p = sg.make_norm_problem(40, channels, dtype, out_dtype="e4m3", scale_group=group)
    y, s, scale = ([torch.zeros_like(t) for t in ts] for ts in (c.out, c.sum, c.out_scale))
    sg.sg_tile_residual_norm(p, c.x, c.weight, y, residual=c.residual, sum_out=s, out_scale=scale)
    torch.cuda.synchronize()
    for i in range(2):
        assert same(s[i], c.sum[i])
        assert bool(((scale[i] - c.out_scale[i]).abs() <= 2.0 ** -18 * scale[i]).all())   # two fp32 maxima, each within a norm's roundings
        _, _, ref, tol = gated64(c.x[i].cpu(), c.residual[i].cpu(), None, None, c.weight.cpu(), None, None, "rms", "none", 1.0, 0, 1e-6)
        for got, sc in ((c.out[i], c.out_scale[i]), (y[i], scale[i])):
            check_eight(got, sc, ref, tol, "e4m3", group)
        # the two agree but for values next to the middle between two steps: some 2^-18 of them to either side, of steps 2^-4 apart
        apart = (c.out[i].view(torch.uint8).int() - y[i].view(torch.uint8).int()).abs()
        assert int(apart.max()) <= 1 and float((apart != 0).float().mean()) < 1e-3


@pytest.mark.parametrize("channels", [64, 256, 1536, 5120, 32768])
@pytest.mark.parametrize("far", [0.0, 0.3, 0.49, 0.499, 0.5, 0.501, 0.51, 0.7, 1.0, 10.0, 1000.0])
def test_layer_norms_on_both_sides_of_the_second_pass(channels, far):
    """Rows whose mean is `far` deviations from 0; up to 1/2 mean and variance come from one pass.  There the sums hold |v| and v^2, whose means are below sqrt(1.25) and 1.25
    deviations: the mean is off by 1.12 SUM of one, the variance by 1.25 SUM for its squares and 2 * 0.5 * 1.12 SUM for the mean's square.  Rows farther out: SUM of what
    the first mean leaves, and of its square."""
    x = torch.randn((6, channels), generator=torch.Generator().manual_seed(channels))
    x = (x - x.mean(dim=1, keepdim=True)) / x.std(dim=1, keepdim=True, unbiased=False) + far
    p = sg.make_gated_norm_problem(6, channels, "f32", norm="layer")
    y = torch.empty((6, channels), device="cuda")
    sg.sg_tile_gated_norm(p, [x.cuda()], [y])
    torch.cuda.synchronize()
    d = x.double() - x.double().mean(dim=1, keepdim=True)
    ref = d / (d.square().mean(dim=1, keepdim=True) + float(torch.tensor(1e-6, dtype=torch.float32))).sqrt()
    # 8 roundings: root, reciprocal, products, the factor 1 / channels, the difference (which is one of v here, far + |z| in size)
    tol = (1.19 * SUM + 8 * U32) * ref.abs() + 1.12 * SUM + 4 * U32 * (min(far, 1.0) + ref.abs())
    off = (y.cpu().double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("wrap", [(0, 0, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1), (0, 2 ** 31 - 8, 5)])
def test_positions_that_wrap_around_the_largest_canvas(wrap):
    """The sum of an origin inside the canvas and a token's place passes 31 bits before it wraps."""
    size = (3, 6, 70)
    origin = [tuple(n - 2 if n else 5 for n in wrap), (2, 2 ** 31 - 10, 3)]
    c = test_gpu_rotary.Call(size=size, heads=1, d=64, axes=(20, 22, 22), dtype="f32", wrap=wrap, origin=origin, base=1e30)
    c.run()
    for i in range(2):
        coords = c.coords(i).double()
        x = c.view(c.q[i], "q").cpu().double()
        axis_of = torch.repeat_interleave(torch.arange(3), torch.tensor([n // 2 for n in c.axes]))
        w = (coords[:, axis_of] * c.freq.cpu())[:, None, :]
        a, b = x[..., 0:64:2], x[..., 1:64:2]
        y = torch.stack([a * w.cos() - b * w.sin(), b * w.cos() + a * w.sin()], dim=-1).flatten(-2)
        # positions up to 2^31: a product of 2^31 and a frequency / 2 pi of two roundings in fp64 is off by 2^-21 turns at most, 2^-18 radians
        tol = (a.abs() + b.abs()) * (2.0 ** -18 + 2.0 ** -21 + 3 * U32)
        off = (c.view(c.q_out[i], "q").cpu().double() - y).abs()
        assert bool((off <= torch.stack([tol, tol], dim=-1).flatten(-2)).all()), float((off / torch.stack([tol, tol], dim=-1).flatten(-2)).max())
