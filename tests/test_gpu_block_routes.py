"""Which kernel a rotary, gated norm or linear call takes, by the names of the launches of a trace, each form held against the 64-bit one; the blocks of the
linear layer also under run flags, whose tiles move to other blocks."""
import re

import pytest
import torch

import test_gpu_gated_norm
import test_gpu_int8_linear
import test_gpu_rotary

pytestmark = pytest.mark.gpu


def _kernels(call):
    """(name, template arguments) of the kernels that a call launches."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as trace:
        call()
        torch.cuda.synchronize()
    names = [e.key for e in trace.key_averages()]
    found = [re.search(r"(rotary|gated_norm|int8_linear_rows|int8_linear)_kernel<([^>]*)>", n) for n in names]
    found = sorted((m.group(1), m.group(2).replace(" ", "")) for m in found if m)
    if not found and not any("sg::" in n for n in names):
        pytest.skip("no trace of kernels on this device")
    return found


# rows of a tile, channels, outputs, tiles, kernel and the sizes of its blocks
LINEAR = [(1, 256, 512, 9, "int8_linear_rows", "1,1,4,4"), (1, 256, 2560, 9, "int8_linear_rows", "1,2,3,8"), (5, 256, 512, 9, "int8_linear_rows", "2,2,2,4"),
          (128, 256, 1024, 9, "int8_linear", "64,64,2,2,3"), (256, 384, 2560, 9, "int8_linear", "128,128,2,2,2"), (1500, 256, 4104, 9, "int8_linear", "256,256,2,4,2")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, channels, outputs, tiles, kernel, sizes", LINEAR)
def test_linear_blocks(dtype, rows, channels, outputs, tiles, kernel, sizes):
    c = test_gpu_int8_linear.Call(rows, channels, outputs, dtype, tiles=tiles, gelu=dtype == "f32")
    kind = "unsignedshort" if dtype == "bf16" else "float"
    assert _kernels(c.run) == [(kernel, kind + "," + sizes)]
    c.check([0, tiles - 1])
    for keep in ([1, 0, 0, 1, 0, 1, 1, 0, 1], [0] * 8 + [1], [0] * 9):
        for t in c.back:
            t.fill_(9.0)
        c.run(run=torch.tensor(keep, dtype=torch.uint8, device="cuda"))
        ran = [i for i in range(tiles) if keep[i]]
        c.check(ran[:1] + ran[-1:])
        assert all(bool((c.back[i] == 9.0).all()) for i in range(tiles) if not keep[i])


@pytest.mark.parametrize("dtype, channels, form", [
    ("bf16", 8, "1,false"), ("bf16", 128, "2,false"), ("f32", 256, "2,false"), ("bf16", 264, "1,true"), ("bf16", 512, "1,true"), ("bf16", 1024, "2,true"), ("f32", 1536, "3,true"),
    ("bf16", 5120, "3,true"), ("bf16", 8192, "2,true"), ("f32", 16384, "2,true"), ("bf16", 32768, "4,true"), ("f32", 20000, "4,true")])
@pytest.mark.parametrize("post", ["none", "rms"])
@pytest.mark.parametrize("mods", ["same", "f32"])
def test_gated_norm_forms(dtype, channels, form, post, mods):
    c = test_gpu_gated_norm.Call(7, channels, dtype, norm="layer", post=post, mod_dtype=mods, mod_rows=3)
    t, m = ("unsignedshort" if dtype == "bf16" else "float"), ("unsignedshort" if dtype == "bf16" and mods == "same" else "float")
    assert _kernels(c.run) == [("gated_norm", ",".join([t, m, form, "true" if post == "rms" else "false"]))]
    c.check()
    if channels % 128 == 0 and channels <= 256:   # blocks of 128 channels: 16 lanes side by side
        c = test_gpu_gated_norm.Call(7, channels, dtype, out="e4m3", group=128)
        assert _kernels(c.run)[0][1].split(",")[2:4] == ["1", "false"]
        c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("d, axes, lines, full", [(128, (32, 48, 48), True, True), (128, (16, 16, 32), True, False), (64, (16, 24, 24), False, True), (96, (32, 32, 32), False, False),
                                                  (256, (64, 96, 96), True, True)])
def test_rotary_forms(dtype, layout, d, axes, lines, full):
    c = test_gpu_rotary.Call(heads=5, kv_heads=3, d=d, axes=axes, dtype=dtype, layout=layout, norm=True, token_major=True)
    flags = [layout == "half", lines and dtype == "bf16", full]
    assert _kernels(c.run) == [("rotary", ",".join(["unsignedshort" if dtype == "bf16" else "float"] + [str(f).lower() for f in flags]))]
    c.check()


def test_listed_positions_of_many_tiles():
    """More tiles than a launch has places for, each with positions of its own."""
    test_gpu_rotary.Call(tiles=70, size=(1, 3, 5), heads=3, kv_heads=1, listed=100000, columns=3, token_major=True).run().check()
