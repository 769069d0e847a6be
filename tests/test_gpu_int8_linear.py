"""8-bit integer linear layers of tiles against exact sums in 64 bits, within the roundings behind the sum."""
import pytest
import torch

import paper_2508_17756_amd as sg
from block_util import TORCH, check, linear64, same

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, rows, channels, outputs, dtype="bf16", tiles=1, bias=True, gelu=False, pad=0, seed=0):
        g = torch.Generator().manual_seed(600 + seed)
        self.dtype, self.tiles, self.gelu, self.rows, self.outputs, self.channels = dtype, tiles, gelu, rows, outputs, channels
        self.p = sg.make_int8_linear_problem(rows, channels, outputs, dtype, activation="gelu" if gelu else None)
        self.p.x_stride, self.p.w_stride, self.p.out_stride = channels + 2 * pad, channels + 4 * pad, outputs + pad

        def ints(n, stride):   # what lies between the rows is not to be read as channels
            t = torch.randint(-128, 128, (n, stride), generator=g, dtype=torch.int8).cuda()
            return t[:, :channels]

        self.x = [ints(rows, self.p.x_stride) for _ in range(tiles)]
        self.w = ints(outputs, self.p.w_stride)
        self.x_scale = [(0.5 + torch.rand(rows, generator=g)).cuda() / 70 for _ in range(tiles)]
        self.w_scale = ((0.5 + torch.rand(outputs, generator=g)) / 70 / channels ** 0.5).cuda()
        self.bias = torch.randn(outputs, generator=g).to(TORCH[dtype]).cuda() if bias else None
        self.back = [torch.full((rows, self.p.out_stride), 9.0, dtype=TORCH[dtype], device="cuda") for _ in range(tiles)]
        self.out = [t[:, :outputs] for t in self.back]

    def run(self, **kw):
        sg.sg_tile_int8_linear(self.p, self.x, self.x_scale, self.w, self.w_scale, self.out, **{"bias": self.bias, **kw})
        torch.cuda.synchronize()
        return self

    def check(self, tiles=None, rows=None):
        at = slice(None) if rows is None else rows
        for i in range(self.tiles) if tiles is None else tiles:
            ref, tol = linear64(self.x[i][at].cpu(), self.x_scale[i][at].cpu(), self.w.cpu(), self.w_scale.cpu(),
                                None if self.bias is None else self.bias.cpu(), self.gelu)
            check(self.out[i][at], ref, tol, self.dtype)
            assert bool((self.back[i][:, self.outputs:] == 9.0).all())
        return self


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 130, 257])
@pytest.mark.parametrize("channels, outputs", [(16, 8), (48, 40), (64, 64), (112, 136), (128, 128), (144, 264), (640, 72), (1040, 520)])
def test_sizes(dtype, rows, channels, outputs):
    Call(rows, channels, outputs, dtype, seed=rows).run().check()
    Call(rows, channels, outputs, dtype, tiles=3, bias=False, pad=16, gelu=True, seed=rows + 1).run().check()


@pytest.mark.parametrize("rows, channels, outputs, tiles", [
    (1, 5120, 640, 20), (3, 16, 2000, 70), (300, 1024, 1000, 4), (1, 20480, 64, 1), (16, 20480, 200, 2), (700, 96, 2568, 3), (2000, 256, 768, 2),
    (1000, 1296, 1032, 5)])
def test_tiles(rows, channels, outputs, tiles):
    for dtype in ("bf16", "f32"):
        Call(rows, channels, outputs, dtype, tiles=tiles).run().check(sorted({0, tiles // 2, tiles - 1}))


def test_large_calls():
    """The blocks of large calls, with ragged ends in rows, channels and outputs."""
    for rows, channels, outputs, tiles, gelu in ((5000, 1040, 2056, 1, True), (1111, 656, 4104, 5, False), (4097, 128, 4096, 2, False), (2500, 2064, 3336, 2, True)):
        c = Call(rows, channels, outputs, tiles=tiles, gelu=gelu, pad=16).run()
        c.check([0, tiles - 1])


def test_the_largest_sum():
    """131,056 channels of -128 * -128: 2^31 - 2^18."""
    for rows in (1, 40, 300):
        c = Call(rows, 131056, 40, "f32", bias=False)
        c.x[0].fill_(-128)
        c.w.fill_(-128)
        c.w[1::2].fill_(127)
        c.x_scale[0].fill_(1.0)
        c.w_scale.fill_(1.0)
        c.run()
        assert bool((c.out[0][:, 0::2] == 131056.0 * 16384).all()) and bool((c.out[0][:, 1::2] == float(torch.tensor(-131056.0 * 16256, dtype=torch.float32))).all())


@pytest.mark.parametrize("rows", [1, 5, 40, 200])
def test_tiles_that_do_not_run_stay(rows):
    flags = torch.arange(70) % 3 != 1
    for keep in (flags, torch.zeros(70, dtype=torch.bool), torch.arange(70) == 69):
        c = Call(rows, 208, 72, tiles=70).run(run=keep.to(torch.uint8).cuda())
        c.check([i for i in range(70) if keep[i]])
        for i in range(70):
            assert keep[i] or bool((c.back[i] == 9.0).all())


@pytest.mark.parametrize("rows", [1, 30, 300])
def test_nan_scales_stay_with_their_rows_and_outputs(rows):
    c = Call(rows, 256, 136)
    c.x_scale[0][rows // 2] = float("nan")
    c.w_scale[7] = float("nan")
    c.run()
    bad = torch.isnan(c.out[0]).cpu()
    want = torch.zeros_like(bad)
    want[rows // 2] = True
    want[:, 7] = True
    assert torch.equal(bad, want)


def test_gelu_of_large_and_small_numbers():
    c = Call(33, 64, 64, "f32", gelu=True, bias=False)
    for gain in (1e-20, 1.0, 30.0, 1e4, 1e12):
        c.w_scale.fill_(gain / 20000)
        c.run().check()


def test_rows_beyond_four_gigabytes():
    stride = (1 << 31) + 64
    for rows in (2, 140):
        c = Call(rows, 64, 64)
        wide = torch.zeros(stride + 64, dtype=torch.int8, device="cuda")
        x = c.w.clone()
        c.w = wide.as_strided((2, 64), (stride, 1))
        c.w.copy_(x[:2])
        c.p.w_stride, c.p.outputs = stride, 8
        full = torch.zeros(7 * stride + 64, dtype=torch.int8, device="cuda").as_strided((8, 64), (stride, 1))
        full.copy_(x[:8])
        c.w, c.w_scale, c.bias, c.outputs = full, c.w_scale[:8].contiguous(), c.bias[:8].contiguous(), 64
        c.run()
        ref, tol = linear64(c.x[0].cpu(), c.x_scale[0].cpu(), full.cpu(), c.w_scale.cpu(), c.bias.cpu(), False)
        check(c.out[0][:, :8], ref, tol, "bf16")
        assert bool((c.out[0][:, 8:] == 9.0).all())
        del full, wide, c
        torch.cuda.empty_cache()


def test_same_bits_every_time_and_captured():
    for rows, channels, outputs in ((1, 5120, 640), (70, 1040, 328), (600, 656, 1032)):
        eager, graphed = (Call(rows, channels, outputs, tiles=2, gelu=True) for _ in range(2))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphed.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            sg.sg_tile_int8_linear(graphed.p, graphed.x, graphed.x_scale, graphed.w, graphed.w_scale, graphed.out, bias=graphed.bias)
        for step in range(3):
            for c in (eager, graphed):
                for t in c.x:
                    t.copy_(t.roll(1, dims=0) if step else t)
                for t in c.x_scale:
                    t.mul_(1.25)
            eager.run()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(eager.out, graphed.out):
                assert same(a, b)


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_behind_the_norm_that_writes_its_integers(out):
    g = torch.Generator().manual_seed(8)
    rows, c, outputs = 75, 640, 200
    x = torch.randn((rows, c), generator=g).to(TORCH[out]).cuda()
    w = torch.randint(-127, 128, (outputs, c), generator=g, dtype=torch.int8).cuda()
    w_scale = torch.rand(outputs, generator=g).cuda() / 1000
    pn = sg.make_gated_norm_problem(rows, c, out, out_dtype="int8", norm="layer")
    q, scale = torch.empty((rows, c), dtype=torch.int8, device="cuda"), torch.empty((rows, 1), device="cuda")
    sg.sg_tile_gated_norm(pn, [x], [q], out_scale=[scale])
    p = sg.make_int8_linear_problem(rows, c, outputs, out)
    y = torch.empty((rows, outputs), dtype=TORCH[out], device="cuda")
    sg.sg_tile_int8_linear(p, [q], [scale], w, w_scale, [y])
    torch.cuda.synchronize()
    ref, tol = linear64(q.cpu(), scale.cpu().flatten(), w.cpu(), w_scale.cpu(), None, False)
    check(y, ref, tol, out)
