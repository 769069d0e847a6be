"""Calls of more workgroups than a grid may have threads for are refused before anything is launched (host only).  Where there is no device, the calls
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
