"""Sums in place, on the host: a buffer that another tile reads or writes meanwhile is refused before anything is launched.  Where there is no device,
the calls that pass the checks end with its error; where there is one, nothing here runs (the addresses are made up)."""
import ctypes

import pytest
import torch

import paper_2508_17756_amd as sg

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="calls that are not refused would be launched")


def _norm(x, residual, total, **fields):
    """Status of a call whose buffers are numbered."""
    p, n = sg.make_norm_problem(5, 256, "bf16"), len(x)
    for name, value in fields.items():
        setattr(p, name, value)
    arr = lambda at: None if at is None else (ctypes.c_void_p * n)(*[0x10000 * (1 + i) for i in at])   # noqa: E731
    return sg.load_library().sg_tile_residual_norm(ctypes.byref(p), n, arr(x), arr(residual), None, None, arr(total), arr(range(1000, 1000 + n)),
                                                   None, None)


@pytest.mark.parametrize("x, residual, total, fields", [
    ([0, 1, 2], [9, 9, 9], [9, 8, 7], {}),            # the residual of all tiles is one of the sums
    ([0, 0, 0], [4, 5, 6], [0, 1, 2], {}),            # so is the input of all
    ([0, 1, 2], [3, 4, 5], [1, 10, 11], {}),          # the input of another tile
    ([0, 1, 2], [3, 4, 5], [10, 11, 10], {}),         # two sums in one place
    ([0, 1, 2], None, [0, 1, 2], {"sum_stride": 512}),        # in place with another stride
    ([0, 1, 2], [3, 4, 5], [3, 4, 5], {"residual_stride": 512}),
    (list(range(256)), None, list(range(255, 511)), {}),
])
def test_sums_where_another_tile_works_are_refused(x, residual, total, fields):
    assert _norm(x, residual, total, **fields) == sg.SG_ERR_INVALID_ARG


@pytest.mark.parametrize("x, residual, total, fields", [
    ([0, 1, 2], [3, 4, 5], [0, 1, 2], {}), ([0, 1, 2], [3, 4, 5], [3, 4, 5], {}), ([0, 1, 2], [9, 9, 9], [0, 1, 2], {}),
    ([0, 1, 2], [0, 1, 2], [0, 1, 2], {}), ([0, 0, 0], [9, 9, 9], [1, 2, 3], {}), ([0, 1, 2], None, [7, 1, 8], {}),
    ([0, 1, 2], [3, 4, 5], [3, 1, 10], {}), ([2, 1, 0], [3, 4, 5], [10, 11, 12], {"sum_stride": 512}), (list(range(256)), None, list(range(256)), {}),
])
def test_sums_in_place_and_apart_are_not(x, residual, total, fields):
    assert _norm(x, residual, total, **fields) == sg.SG_ERR_HIP
