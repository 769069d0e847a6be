"""Limits of the context attentions, host only: calls of more workgroups than a grid may have threads for, and with too small a workspace, are refused
before anything is launched.  Where there is no device, the calls
that pass the checks end with its error; where there is one, nothing here runs (the addresses are made up)."""
import ctypes

import pytest
import torch

import paper_2508_17756_amd as sg

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="calls that are not refused would be launched")


@pytest.mark.parametrize("dtype, tiles, tokens, heads, status", [
    ("f32", 64, 257, 65535, sg.SG_ERR_UNSUPPORTED),    # 5 blocks of 64 queries: 20,971,200
    ("f32", 130, 257, 65535, sg.SG_ERR_UNSUPPORTED),   # (of its largest launch)
    ("f32", 64, 256, 65535, sg.SG_ERR_HIP),            # 4: 16,776,960
    ("f32", 51, 257, 65535, sg.SG_ERR_HIP),            # 16,711,425
    ("f32", 52, 257, 65535, sg.SG_ERR_UNSUPPORTED),    # 17,039,100
    ("bf16", 64, 32767, 1024, sg.SG_ERR_UNSUPPORTED),  # 256 blocks of 128 queries: 2^24
    ("bf16", 64, 32767, 1023, sg.SG_ERR_HIP),
])
def test_more_workgroups_than_a_grid_takes(dtype, tiles, tokens, heads, status):
    p = sg.make_context_problem(tokens, 5000, heads, 64, dtype)
    a = (ctypes.c_void_p * tiles)(*[0x10000] * tiles)
    lib = sg.load_library()
    assert lib.sg_context_validate(ctypes.byref(p)) == sg.SG_OK
    assert lib.sg_tile_cross_attention(ctypes.byref(p), tiles, a, a, a, None, None, None, a, None, 0, None) == status


def _refused(p, tiles, prefix, size):
    a, lib = (ctypes.c_void_p * tiles)(*[0x10000] * tiles), sg.load_library()
    if prefix:
        st = lib.sg_tile_prefix_attention(ctypes.byref(p), tiles, a, a, a, 0x10000, 0x10000, None, None, None, a, 0x10000, size, None)
    else:
        st = lib.sg_tile_cross_attention(ctypes.byref(p), tiles, a, a, a, None, None, None, a, 0x10000, size, None)
    assert st in (sg.SG_ERR_WORKSPACE, sg.SG_ERR_HIP)
    return st == sg.SG_ERR_WORKSPACE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_each_call_needs_its_own_workspace_to_the_last_byte(dtype):
    # keys of the tiles alone: the cross attention has none, so that the size is the prefix attention's
    p = sg.make_context_problem(1, 0, 8, 128, dtype, own_tokens=30000)
    need = sg.sg_context_workspace_bytes(p, 2)
    assert need > 0 and _refused(p, 2, True, need - 1) and not _refused(p, 2, True, need) and not _refused(p, 2, False, 0)
    # one tile whose keys are all the prefix's: the two calls are the same
    p = sg.make_context_problem(1, 30000, 8, 128, dtype)
    need = sg.sg_context_workspace_bytes(p, 1)
    for prefix in (False, True):
        assert need > 0 and _refused(p, 1, prefix, need - 1) and not _refused(p, 1, prefix, need)
    # more tiles than a launch takes: the largest launch's, here the last one, whose two tiles are cut further than 64
    p = sg.make_context_problem(40, 30000, 8, 128, dtype)
    need = sg.sg_context_workspace_bytes(p, 66)
    assert need >= max(sg.sg_context_workspace_bytes(p, n) for n in (2, 64))
    assert need > 0 and _refused(p, 66, False, need - 1) and not _refused(p, 66, False, need)
