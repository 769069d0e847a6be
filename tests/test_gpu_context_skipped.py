"""Tiles that do not run take little time of a context attention whose work fills the device (the workgroups that are left are spread over all of it),
and of a residual norm."""
import statistics

import pytest
import torch

import paper_2508_17756_amd as sg
from context_util import TORCH, Call

pytestmark = pytest.mark.gpu


def _time(call):
    """Microseconds of a call, median of 9 runs of 10."""
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    took = []
    for _ in range(12):
        start.record()
        for _ in range(10):
            call()
        end.record()
        torch.cuda.synchronize()
        took.append(start.elapsed_time(end) * 100.0)
    return statistics.median(took[3:])


@pytest.mark.parametrize("dtype, d, tokens, heads, ctx", [("f32", 128, 2880, 8, 226), ("f32", 64, 2880, 16, 226), ("bf16", 128, 3840, 24, 512),
                                                          ("bf16", 64, 3840, 24, 900), ("bf16", 64, 9000, 24, 226)])
def test_half_of_the_tiles_take_about_half_of_the_time(dtype, d, tokens, heads, ctx):
    """8 tiles: any 4 of them less than 3/4, one less than a third of what all take."""
    c = Call(8, tokens, heads, heads, d, dtype, ctx)
    ws = c.workspace()

    def took(run):
        flags = torch.tensor(run, dtype=torch.uint8, device="cuda")
        return _time(lambda: sg.sg_tile_cross_attention(c.p, c.q, c.k, c.v, c.out, run=flags, workspace=ws))

    whole = took([1] * 8)
    for run in ([1, 1, 1, 1, 0, 0, 0, 0], [0, 0, 0, 0, 1, 1, 1, 1], [1, 0, 1, 0, 1, 0, 1, 0]):
        assert took(run) < 0.75 * whole, run
    for one in (0, 5):
        assert took([int(i == one) for i in range(8)]) < whole / 3, one


@pytest.mark.parametrize("channels, rows, dtype, out", [(5120, 9450, "bf16", "e4m3"), (5120, 9450, "bf16", None), (768, 60000, "bf16", None),
                                                        (4096, 6000, "f32", None), (30720, 1500, "bf16", None)])
def test_rows_of_tiles_that_do_not_run_take_little_time(channels, rows, dtype, out):
    """8 tiles: none of them less than a quarter, any 4 of them less than 0.7 of what all take."""
    dt = TORCH[dtype]
    x, r, total = ([torch.randn((rows, channels), device="cuda").to(dt) for _ in range(8)] for _ in range(3))
    y = [torch.empty((rows, channels), dtype=torch.float8_e4m3fn if out else dt, device="cuda") for _ in range(8)]
    scale = [torch.empty((rows, 1), device="cuda") for _ in range(8)] if out else None
    w = torch.ones(channels, device="cuda").to(dt)
    p = sg.make_norm_problem(rows, channels, dtype, out_dtype=out)

    def took(run):
        flags = torch.tensor(run, dtype=torch.uint8, device="cuda")
        return _time(lambda: sg.sg_tile_residual_norm(p, x, w, y, residual=r, sum_out=total, out_scale=scale, run=flags))

    whole = took([1] * 8)
    assert took([0] * 8) < 0.25 * whole
    assert took([1, 0] * 4) < 0.7 * whole and took([0, 0, 0, 0, 1, 1, 1, 1]) < 0.7 * whole
