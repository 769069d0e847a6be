"""Norms with gate, residual scale and modulation against the formula in 64 bits, within the roundings the kernel makes."""
import itertools

import pytest
import torch

import paper_2508_17756_amd as sg
from block_util import TORCH, check, check_eight, gated64, same

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, rows, channels, dtype="bf16", tiles=2, out="same", group=0, norm="rms", post="none", residual=True, gate=True, mod=True, weight=False,
                 post_weight=None, mod_rows=0, mod_dtype="same", residual_scale=1.0, total=True, pad=0, gain=1.0, around=0.0, eps=1e-6, seed=0):
        g = torch.Generator().manual_seed(500 + seed)
        dt = TORCH[dtype]
        mt = dt if mod_dtype == "same" else torch.float32
        self.rows, self.channels, self.dtype, self.out_kind, self.group, self.norm, self.post = rows, channels, dtype, out, group, norm, post
        self.mod_rows, self.residual_scale, self.tiles, self.eps = mod_rows, residual_scale, tiles, eps
        self.p = sg.make_gated_norm_problem(rows, channels, dtype, out_dtype=None if out == "same" else out, scale_group=group, norm=norm, post_norm=post,
                                            residual_scale=residual_scale, mod_rows=mod_rows, mod_dtype=None if mod_dtype == "same" else "f32", eps=eps,
                                            post_eps=eps)
        for name in ("x", "residual", "sum", "out", "mod"):
            setattr(self.p, name + "_stride", channels + pad)

        def tensor(n, kind, size=1.0, at=0.0):
            t = torch.zeros((n, channels + pad), dtype=kind).cuda()
            t[:, :channels] = (at + size * torch.randn((n, channels), generator=g)).to(kind).cuda()
            return t[:, :channels]

        many = lambda n, kind, **kw: [tensor(n, kind, **kw) for _ in range(tiles)]   # noqa: E731
        vectors = -(-rows // mod_rows) if mod_rows else 1
        self.x = many(rows, dt, size=gain, at=around)
        self.residual = many(rows, dt, size=gain) if residual else None
        self.gate = many(vectors, mt, size=0.5) if gate else None
        self.scale, self.shift = (many(vectors, mt, size=0.3) if mod else None for _ in range(2))
        self.weight = tensor(1, dt, size=0.2, at=1.0)[0] if weight else None
        self.post_weight = tensor(1, dt, size=0.2, at=1.0)[0] if (post != "none" if post_weight is None else post_weight) else None
        blank = lambda kind: [torch.zeros((rows, channels + pad), dtype=kind, device="cuda")[:, :channels] for _ in range(tiles)]   # noqa: E731
        self.sum = blank(dt) if total else None
        self.out = blank({"same": dt, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[out])
        self.out_scale = [torch.full((rows, channels // group if group else 1), -1.0, device="cuda") for _ in range(tiles)] if out != "same" else None

    def run(self, **kw):
        sg.sg_tile_gated_norm(self.p, self.x, self.out, **{**dict(residual=self.residual, gate=self.gate, post_weight=self.post_weight,
                              weight=self.weight, scale=self.scale, shift=self.shift, sum_out=self.sum, out_scale=self.out_scale), **kw})
        torch.cuda.synchronize()
        return self

    def reference(self, i):
        cpu = lambda v: None if v is None else (v[i] if isinstance(v, list) else v).cpu()   # noqa: E731
        return gated64(cpu(self.x), cpu(self.residual), cpu(self.gate), cpu(self.post_weight), cpu(self.weight), cpu(self.scale), cpu(self.shift),
                       self.norm, self.post, self.residual_scale, self.mod_rows, self.eps)

    def check(self, tiles=None):
        for i in range(self.tiles) if tiles is None else tiles:
            s, es, y, ey = self.reference(i)
            if self.sum is not None:
                check(self.sum[i], s, es, self.dtype)
            if self.out_kind == "same":
                check(self.out[i], y, ey, self.dtype)
            else:
                check_eight(self.out[i], self.out_scale[i], y, ey, self.out_kind, self.group)
        return self

    def outputs(self):
        return self.out + (self.sum or []) + (self.out_scale or [])


SIZES = [(1, 8), (3, 16), (5, 40), (7, 64), (9, 128), (4, 136), (6, 256), (5, 504), (5, 512), (3, 520), (3, 1024), (2, 1536), (2, 2048), (2, 2056),
         (3, 4096), (2, 5120), (2, 6000), (2, 8192), (2, 8200), (1, 16384), (1, 20000), (2, 32768)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, channels", SIZES)
def test_sizes(dtype, rows, channels):
    Call(rows, channels, dtype, norm="layer", seed=channels).run().check()
    Call(rows, channels, dtype, norm="rms", post="rms", mod_rows=2, mod_dtype="f32", residual_scale=0.5, pad=8, seed=channels + 1).run().check()
    Call(rows, channels, dtype, norm="layer", post="layer", residual=False, gate=False, mod=False, weight=True, total=False).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["e4m3", "int8"])
@pytest.mark.parametrize("rows, channels", SIZES)
def test_eight_bits(dtype, out, rows, channels):
    Call(rows, channels, dtype, out=out, norm="layer", pad=16, seed=channels).run().check()
    if channels % 128 == 0:
        Call(rows, channels, dtype, out=out, group=128, norm="rms", post="layer", mod_dtype="f32", seed=channels + 2).run().check()


@pytest.mark.parametrize("norm, post", itertools.product(["rms", "layer"], ["none", "rms", "layer"]))
def test_every_choice_of_parts(norm, post):
    for k, (residual, gate, mod, weight, total) in enumerate(itertools.product([False, True], repeat=5)):
        Call(5, 192, "bf16", tiles=1, norm=norm, post=post, residual=residual, gate=gate, mod=mod, weight=weight, total=total, seed=k,
             out="int8" if k % 3 == 0 else "same", residual_scale=-1.5).run().check()
    c = Call(5, 192, "f32", norm=norm, post=post, post_weight=False)
    c.run(scale=None).scale = None
    c.check()
    c = Call(5, 192, "f32", norm=norm, post=post)
    c.run(shift=None).shift = None
    c.check()


@pytest.mark.parametrize("mod_rows", [1, 3, 7, 49, 50, 51, 1000])
def test_rows_that_share_vectors(mod_rows):
    Call(50, 136, "bf16", mod_rows=mod_rows, mod_dtype="f32").run().check()
    Call(50, 2056, "bf16", mod_rows=mod_rows, norm="layer").run().check()
    Call(50, 640, "f32", mod_rows=mod_rows, out="e4m3", group=128).run().check()


def test_rows_beyond_the_grid():
    """More rows than the launch has places for: every workgroup walks several."""
    Call(30011, 128, "bf16", tiles=3, mod_rows=1000).run().check([0, 2])
    Call(4099, 2056, "bf16", out="int8", mod_rows=100, norm="layer").run().check()
    Call(1031, 8200, "f32", tiles=1, out="e4m3").run().check()
    Call(9000, 1024, "bf16", tiles=2, post="rms").run().check()


@pytest.mark.parametrize("channels", [64, 2048, 5120])
def test_tiles_that_do_not_run_stay(channels):
    flags = torch.arange(70) % 3 != 1
    for out in ("same", "int8"):
        c = Call(6, channels, "bf16", tiles=70, out=out).run(run=flags.cuda())
        c.check([i for i in range(70) if flags[i]][::6])
        for i in range(70):
            if not flags[i]:
                assert float(c.out[i].float().abs().max()) == 0 and float(c.sum[i].float().abs().max()) == 0
                assert out == "same" or bool((c.out_scale[i] == -1).all())


@pytest.mark.parametrize("which", ["x", "residual"])
@pytest.mark.parametrize("channels", [128, 5120])
def test_sums_in_place(which, channels):
    apart = Call(33, channels, "bf16", post="rms", norm="layer").run()
    c = Call(33, channels, "bf16", post="rms", norm="layer")
    c.sum = getattr(c, which)
    c.run()
    for a, b in zip(apart.outputs(), c.outputs()):
        assert same(a, b)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("channels", [64, 1024, 5120])
@pytest.mark.parametrize("gain", [1e37, 1e25, 1e-25, 1e-38])
def test_rows_whose_squares_leave_the_range(norm, channels, gain):
    """As the formula says without an eps, also where a sum of squares is beyond 2^128 or below 2^-149.  (1e-38: the values are rounded to multiples of
    2^-149 already in x; differences of two such are exact.)"""
    c = Call(3, channels, "f32", norm=norm, gain=gain, residual=False, gate=False, eps=0.0, total=False).run()
    if gain > 1e-30:
        c.check()
    else:   # the mean of numbers near 2^-126 is rounded to a multiple of 2^-149: 2^-23 of them
        for i in range(2):
            _, _, y, ey = c.reference(i)
            check(c.out[i], y, ey + 2.0 ** -20 * (1 + y.abs()), "f32")
    Call(3, channels, "f32", post=norm, norm="rms", gain=gain, residual=False, eps=0.0).run()


@pytest.mark.parametrize("around", [100.0, -30000.0])
def test_rows_far_from_zero(around):
    """mean(v^2) - mean(v)^2 in fp32 would leave nothing of a deviation of 1 around 30,000; the two means keep it to fp32's own rounding of the values."""
    Call(5, 5120, "f32", norm="layer", around=around, residual=False, gate=False, total=False).run().check()
    Call(5, 256, "f32", norm="layer", post="layer", around=around).run().check()


def test_rows_of_zeros_and_of_one_value():
    for norm in ("rms", "layer"):
        c = Call(4, 640, "f32", norm=norm, residual=False, gate=False, out="int8")
        for t in c.x:
            t.zero_()
        c.run().check()
    c = Call(4, 640, "f32", norm="layer", residual=False, gate=False, mod=False)
    for t in c.x:
        t.fill_(3.0)
    c.run()
    assert all(bool((t == 0).all()) for t in c.out)
    c = Call(4, 640, "f32", norm="layer", residual=False, gate=False, mod=False, out="e4m3")
    for t in c.x:
        t.fill_(-7.0)
    c.run()
    assert all(bool((t.float() == 0).all()) for t in c.out) and all(bool((t == 0).all()) for t in c.out_scale)


@pytest.mark.parametrize("out", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("channels", [64, 640, 5120])
def test_nan_and_infinity_stay_in_their_rows(out, channels):
    for value in (float("nan"), float("inf")):
        for norm in ("rms", "layer"):
            c, clean = (Call(9, channels, "f32", norm=norm, out=out) for _ in range(2))
            c.x[1][4, 5] = value
            c.run()
            clean.run()
            for a, b in zip(c.outputs(), clean.outputs()):
                if a.shape[0] == 9:
                    assert same(a[torch.arange(9) != 4], b[torch.arange(9) != 4])
            assert same(c.out[0], clean.out[0])
            if out != "same":
                assert bool(torch.isnan(c.out_scale[1][4]).all())
            elif norm == "layer" or value != value:
                assert bool(torch.isnan(c.out[1][4]).all())
            else:   # (infinity / infinity there, nothing elsewhere but the shift)
                bad = torch.isnan(c.out[1][4]).cpu()
                assert bool(bad[5]) and int(bad.sum()) == 1
                assert same(torch.cat([c.out[1][4][:5], c.out[1][4][6:]]), torch.cat([c.shift[1][0][:5], c.shift[1][0][6:]]))


def test_an_output_beyond_the_range_has_a_scale_of_nan():
    c = Call(2, 256, "f32", out="e4m3", group=128)
    for t in c.scale:
        t[:, 130] = 3e38
    for t in c.x:
        t[:, 130] = 100.0
    c.run()
    assert bool(torch.isnan(c.out_scale[0][:, 1]).all()) and bool(torch.isfinite(c.out_scale[0][:, 0]).all())


def test_it_is_the_residual_norm_without_gate_and_modulation():
    for out in ("same", "e4m3"):
        c = Call(40, 640, "bf16", gate=False, mod=False, weight=True, out=out)
        c.run().check()
        p = sg.make_norm_problem(40, 640, "bf16", out_dtype=None if out == "same" else out)
        y, s = [torch.zeros_like(t) for t in c.out], [torch.zeros_like(t) for t in c.sum]
        scale = [torch.zeros_like(t) for t in c.out_scale] if out != "same" else None
        sg.sg_tile_residual_norm(p, c.x, c.weight, y, residual=c.residual, sum_out=s, out_scale=scale)
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(s, c.sum))
        if out == "same":   # two roundings of numbers that differ by fp32 roundings only: at most one step apart
            assert all(bool(((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs()).all()) for a, b in zip(y, c.out))


def test_rows_beyond_four_gigabytes():
    rows, stride = 3, (1 << 30) + 64
    c = Call(rows, 64, "bf16", tiles=1, residual=False, total=False)
    big = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((rows, 64), (stride, 1))
    far.copy_(c.x[0])
    c.x, c.p.x_stride = [far], stride
    c.run().check()


def test_on_another_stream_and_captured():
    eager, graphed = (Call(37, 1536, "bf16", norm="layer", post="rms", out="int8", mod_rows=10) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        sg.sg_tile_gated_norm(graphed.p, graphed.x, graphed.out, residual=graphed.residual, gate=graphed.gate, post_weight=graphed.post_weight,
                              scale=graphed.scale, shift=graphed.shift, sum_out=graphed.sum, out_scale=graphed.out_scale)
    for step in range(3):
        for c in (eager, graphed):
            for t in c.x + c.gate:
                t.mul_(-0.5 - step)
        eager.run()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.outputs(), graphed.outputs()):
            assert same(a, b)
