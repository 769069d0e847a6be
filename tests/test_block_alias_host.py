"""Buffers that gated norms and 8-bit integer linear layers write and that are written or read in another place too are refused, on the host (no GPU is touched here)."""
import pytest

from test_block_host import BAD, DONE, GOOD, _at, _linear, _list, _norm, no_device

EIGHT = {"out_dtype": 3}
PLACE = GOOD + 4096 * 50   # in nobody's list unless it is put there


@pytest.mark.parametrize("places", [[700, 700], [0, 701], [1, 701], [101, 701], [200, 701], [301, 701], [700, 400], [500, 701], [501, 700], [600, 701], [601, 700]])
@pytest.mark.parametrize("group", [0, 128])
def test_scales_of_a_norm_in_a_place_that_has_a_use(places, group):
    """Twice, or where x, residual, gate, scale, shift, sum or out is."""
    assert _norm(fields={**EIGHT, "scale_group": group}, out_scale=places) == BAD


def test_what_a_norm_writes_where_its_weights_are():
    for kw in (dict(weight=PLACE), dict(post_weight=PLACE)):
        assert _norm(out=[50, 601], **kw) == BAD
        assert _norm(total=[500, 50], **kw) == BAD
        assert _norm(fields=EIGHT, out_scale=[50, 701], **kw) == BAD


@no_device
def test_norms_whose_buffers_lie_apart():
    assert _norm(fields=EIGHT, out_scale=[700, 701], weight=PLACE, post_weight=PLACE) == DONE
    assert _norm(fields=EIGHT, out_scale=[700, 701], total=[0, 1]) == DONE
    assert _norm(out_scale=None, total=[100, 101], weight=PLACE) == DONE


@pytest.mark.parametrize("kw", [dict(x_scale=_list([600, 301])), dict(x_scale=_list([300, 600])), dict(w=PLACE, out=_list([600, 50])), dict(w_scale=PLACE, out=_list([50, 601])),
                                dict(bias=PLACE, out=_list([50, 601]))])
def test_linear_results_in_a_place_that_is_read(kw):
    assert _linear(**kw) == BAD


@no_device
def test_linear_results_that_lie_apart():
    assert _linear(w=PLACE, w_scale=PLACE, bias=PLACE) == DONE
    assert _linear(x_scale=_at(2, 300), bias=None, out=_list([50, 51])) == DONE
