"""Residual addition and root-mean-square norm against the formula in 64 bits, within the roundings the kernel makes."""
import pytest
import torch

import paper_2508_17756_amd as sg
from context_util import TORCH, U8, U16, U32, norm64

pytestmark = pytest.mark.gpu


def _call(tiles, rows, channels, dtype, out_dtype=None, group=0, residual=True, weight=True, total=True, pad=0, seed=0, run=None, gain=1.0):
    g = torch.Generator().manual_seed(77 + seed)
    dt = TORCH[dtype]
    p = sg.make_norm_problem(rows, channels, dtype, out_dtype=out_dtype, scale_group=group)

    def rows_of(kind):
        x = torch.full((rows, channels + pad), float("nan") if kind is not torch.uint8 else 0).to(dt) if kind is None else \
            torch.zeros((rows, channels + pad), dtype=kind)
        return x.to("cuda")[:, :channels]

    def values():
        t = rows_of(None)
        t.copy_((torch.randn((rows, channels), generator=g) * gain).to(dt))
        return t

    x = [values() for _ in range(tiles)]
    r = [values() for _ in range(tiles)] if residual else None
    w = (1 + 0.2 * torch.randn((channels,), generator=g)).to(dt).to("cuda") if weight else None
    s = [torch.zeros_like(t) for t in x] if total else None
    if total and pad:
        s = [rows_of(None) for _ in x]
    out = [rows_of(torch.float8_e4m3fn if out_dtype else dt) for _ in x]
    scale = [torch.full((rows, channels // group if group else 1), -1.0, device="cuda") for _ in x] if out_dtype else None
    for name in ("x", "residual", "sum", "out"):
        setattr(p, name + "_stride", channels + pad)
    sg.sg_tile_residual_norm(p, x, w, out, residual=r, sum_out=s, out_scale=scale, run=run)
    torch.cuda.synchronize()
    return p, x, r, w, s, out, scale


def _check(p, x, r, w, s, out, scale, dtype, group=0, tiles=None):
    """s: one rounding of an fp32 sum.  y: the sum of squares is off by (channels / 2 + 8) 2^-24 of itself at most, the root, its reciprocal and the
    two products by 8 roundings, then the store.  8 bits: half a step of 2^-3, or of 2^-9 below the smallest normal number."""
    c = x[0].shape[1]
    u = U16 if dtype == "bf16" else U32
    for i in range(len(x)) if tiles is None else tiles:
        total, y = norm64(x[i].cpu(), None if r is None else r[i].cpu(), None if w is None else w.cpu(), 1e-6)
        mag = x[i].cpu().double().abs() + (0 if r is None else r[i].cpu().double().abs())
        if s is not None:
            assert bool(((s[i].cpu().double() - total).abs() <= u * total.abs() + U32 * mag + 1e-30).all())
        rel = (c / 4 + 16) * U32
        # a sum that cancels keeps the absolute error of its terms
        tol = rel * y.abs() + 2 * U32 * (y / total.where(total != 0, torch.ones_like(total))).abs() * mag
        got = out[i].cpu()
        if scale is None:
            assert bool(((got.double() - y).abs() <= tol + u * y.abs() * (1 + 2 * rel) + 1e-30).all())
            continue
        sc = scale[i].cpu().double()
        blocks = y.reshape(y.shape[0], -1, group or c)
        most = blocks.abs().amax(dim=-1)
        tol_most = tol.reshape(blocks.shape).amax(dim=-1) + 4 * U32 * most
        assert bool(((sc * 448 - most).abs() <= tol_most + 1e-30).all())
        deq = got.float().double().reshape(blocks.shape) * sc[..., None]
        assert bool(torch.isfinite(deq).all())
        assert bool(((deq - blocks).abs() <= tol.reshape(blocks.shape) * (1 + U8) + (U8 + 8 * U32) * blocks.abs() + 2.0 ** -10 * sc[..., None] + 1e-30).all())


SIZES = [(1, 8), (3, 16), (5, 40), (7, 64), (9, 128), (4, 136), (6, 256), (5, 504), (5, 512), (3, 520), (3, 1024), (2, 1536), (2, 2048), (2, 2056),
         (3, 4096), (2, 5120), (2, 6000), (2, 8192), (2, 8200), (1, 16384), (1, 20000), (2, 32768)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, channels", SIZES)
def test_sizes(dtype, rows, channels):
    _check(*_call(2, rows, channels, dtype, seed=channels), dtype)
    _check(*_call(1, rows, channels, dtype, residual=False, weight=False, total=False, pad=8, seed=channels + 1), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, channels", SIZES)
def test_eight_bits(dtype, rows, channels):
    _check(*_call(2, rows, channels, dtype, out_dtype="e4m3", pad=16, seed=channels), dtype)
    if channels % 128 == 0:
        _check(*_call(2, rows, channels, dtype, out_dtype="e4m3", group=128, residual=False, seed=channels), dtype, group=128)


@pytest.mark.parametrize("channels", [64, 128, 2048, 5120])
def test_many_rows_and_skipped_tiles(channels):
    rows = 40000 if channels <= 128 else 700
    run = torch.tensor([1, 0, 1, 1, 0] * 14, dtype=torch.uint8)[:5 if channels > 128 else 67].to("cuda")
    tiles = run.numel()
    rows = rows if tiles == 5 else 1000
    for kw in ({}, {"out_dtype": "e4m3"}):
        got = _call(tiles, rows, channels, "bf16", run=run, **kw)
        keep = [i for i in range(tiles) if run[i]]
        _check(*got, "bf16", tiles=keep[:6] + keep[-2:])
        for i in range(tiles):
            if not run[i]:
                assert float(got[4][i].abs().max()) == 0 and float(got[5][i].float().abs().max()) == 0
                assert got[6] is None or float(got[6][i].max()) == -1


def test_rows_beyond_the_grid():
    """More rows than the launch has places for: every workgroup walks several."""
    _check(*_call(3, 30011, 128, "bf16", residual=False, seed=1), "bf16")
    _check(*_call(2, 4099, 2056, "bf16", out_dtype="e4m3", seed=2), "bf16")
    _check(*_call(1, 1031, 8200, "f32", out_dtype="e4m3", seed=3), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", [128, 5120])
def test_in_place(dtype, channels):
    for which in ("x", "residual"):
        g = torch.Generator().manual_seed(5)
        x, r = (torch.randn((33, channels), generator=g).to(TORCH[dtype]).cuda() for _ in range(2))
        p = sg.make_norm_problem(33, channels, dtype)
        s, y = torch.empty_like(x), torch.empty_like(x)
        sg.sg_tile_residual_norm(p, [x], None, [y], residual=[r], sum_out=[s])
        x2, r2, y2 = x.clone(), r.clone(), torch.empty_like(x)
        sg.sg_tile_residual_norm(p, [x2], None, [y2], residual=[r2], sum_out=[x2 if which == "x" else r2])
        torch.cuda.synchronize()
        assert torch.equal(x2 if which == "x" else r2, s) and torch.equal(y, y2)


def test_zeros_tiny_large_and_nan_rows():
    for channels in (128, 1024, 5120, 9000):
        for dtype in ("bf16", "f32"):
            x = torch.randn((6, channels), generator=torch.Generator().manual_seed(3)).to(TORCH[dtype]).cuda()
            x[0] = 0
            x[1] *= 1e-18
            x[2] *= 2.0 ** 50
            x[3, channels // 2] = float("nan")
            for kw, y in (({}, torch.empty_like(x)), ({"out_dtype": "e4m3"}, torch.empty((6, channels), dtype=torch.float8_e4m3fn, device="cuda"))):
                p = sg.make_norm_problem(6, channels, dtype, **kw)
                scale = [torch.empty((6, 1), device="cuda")] if kw else None
                sg.sg_tile_residual_norm(p, [x], None, [y], out_scale=scale)
                torch.cuda.synchronize()
                got = y.float().cpu()
                assert float(got[0].abs().max()) == 0
                assert bool(torch.isnan(got[3]).all())
                for row in (1, 2, 4, 5):
                    assert bool(torch.isfinite(got[row]).all())
                if not kw:
                    _, want = norm64(x[[1, 2, 4]].cpu(), None, None, 1e-6)
                    assert float((got[[1, 2, 4]].double() - want).abs().max()) < (2.0 ** -8 + 1e-4) * float(want.abs().max())


def test_replays_from_a_graph():
    g = torch.Generator().manual_seed(6)
    x, r = (torch.randn((50, 2048), generator=g).bfloat16().cuda() for _ in range(2))
    p = sg.make_norm_problem(50, 2048, "bf16", out_dtype="e4m3")
    y = [torch.zeros((50, 2048), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    sc = [torch.zeros((50, 1), device="cuda") for _ in range(2)]
    s = [torch.zeros_like(x) for _ in range(2)]
    call = lambda i: sg.sg_tile_residual_norm(p, [x], None, [y[i]], residual=[r], sum_out=[s[i]], out_scale=[sc[i]])   # noqa: E731
    call(0)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(1)
    torch.cuda.synchronize()
    for k in range(3):
        x.mul_(0.5 + k)
        call(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y[0].view(torch.uint8), y[1].view(torch.uint8)) and torch.equal(s[0], s[1]) and torch.equal(sc[0], sc[1])
