"""Gated norms of more rows than a launch has workgroups for (2^21, each of one long row or of up to 256 short ones): workgroups go on to further rows, of another tile,
with the vectors of that tile, also where the tile of their first row does not run."""
import pytest
import torch

import paper_2508_17756_amd as sg
from block_util import TORCH, check, check_eight, gated64

pytestmark = pytest.mark.gpu

WORKGROUPS, PERIOD, TILES = 1 << 21, 1000, 3


@pytest.mark.parametrize("rows, channels, rows_per_workgroup, dtype, out, norm, post", [
    (750_000, 264, 1, "bf16", "same", "rms", "none"),        # a wavefront a row, gate, scale and shift behind one another in LDS
    (750_000, 1544, 1, "bf16", "int8", "layer", "layer"),    # two wavefronts that meet for every sum and maximum
    (750_000, 520, 1, "f32", "e4m3", "layer", "none"),
    (200_000_000, 8, 256, "bf16", "same", "layer", "none"),  # a lane a row
    (12_000_000, 256, 16, "bf16", "int8", "rms", "none")])   # 16 lanes a row
def test_workgroups_go_on_to_further_rows(rows, channels, rows_per_workgroup, dtype, out, norm, post):
    assert rows * TILES > WORKGROUPS * rows_per_workgroup > rows * (TILES - 1) and rows % PERIOD == 0
    g = torch.Generator().manual_seed(channels)
    dt = TORCH[dtype]
    kind = {"same": dt, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[out]
    rnd = lambda n, size: (size * torch.randn((n, channels), generator=g)).to(dt).cuda()   # noqa: E731
    base = rnd(PERIOD, 1.0)
    x = base.repeat(rows // PERIOD, 1)   # what all tiles read
    gate, scale, shift = ([rnd(1, 0.5) for _ in range(TILES)] for _ in range(3))
    y = [torch.empty((rows, channels), dtype=kind, device="cuda") for _ in range(TILES)]
    y_scale = [torch.empty((rows, 1), device="cuda") for _ in range(TILES)] if out != "same" else None
    p = sg.make_gated_norm_problem(rows, channels, dtype, out_dtype=None if out == "same" else out, norm=norm, post_norm=post)
    for run in ([1, 1, 1], [0, 1, 1], [1, 0, 0]):
        for t in y:
            t.view(torch.uint8).fill_(7)
        for t in y_scale or []:
            t.fill_(-1.0)
        sg.sg_tile_gated_norm(p, [x] * TILES, y, gate=gate, scale=scale, shift=shift, out_scale=y_scale, run=torch.tensor(run, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        for i in range(TILES):
            if not run[i]:
                assert bool((y[i].view(torch.uint8) == 7).all()) and (y_scale is None or bool((y_scale[i] == -1).all()))
                continue
            for t in [y[i]] + ([y_scale[i]] if y_scale else []):   # a row has the bits that it has in the first period
                bits = t.view(torch.uint8).view(rows // PERIOD, PERIOD, -1)
                assert torch.equal(bits, bits[:1].expand_as(bits)), (i, run)
            few = slice(0, PERIOD, 37)
            _, _, ref, tol = gated64(base[few].cpu(), None, gate[i].cpu(), None, None, scale[i].cpu(), shift[i].cpu(), norm, post, 1.0, 0, 1e-6)
            if out == "same":
                check(y[i][:PERIOD][few], ref, tol, dtype)
            else:
                check_eight(y[i][:PERIOD][few], y_scale[i][:PERIOD][few], ref, tol, out, 0)
