"""Lengths, masks and run flags that the binding hands to the library, on the host: what the library would read as other values is refused."""
import pytest
import torch

import paper_2508_17756_amd as sg
from paper_2508_17756_amd import binding


class _Host:
    """A tensor's stand-in for the binding."""

    def data_ptr(self):
        return 0x10000


class _Device:
    """A device vector's stand-in for the binding: a tensor on the host that says that it is not."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_lengths_masks_and_flags_of_another_kind_are_refused():
    """The library reads 32-bit lengths and one byte for each place and tile, side by side in device memory: anything else would be other values
    (int64 lengths: every second tile 0), or memory behind the vector."""
    # (problems that the library refuses: nothing is launched whatever the binding lets through)
    p, n, two = sg.make_context_problem(12, 20, 4, 64, "bf16", own_tokens=12), sg.make_norm_problem(5, 256, "bf16"), [_Host()] * 2
    p.scale, n.eps = 0.0, -1.0
    calls = {
        "ctx_len": (lambda t: sg.sg_tile_cross_attention(p, two, two, two, two, ctx_len=t), torch.int32, 2),
        "key_mask": (lambda t: sg.sg_tile_cross_attention(p, two, two, two, two, key_mask=t), torch.uint8, 2 * p.ctx_tokens),
        "cross_run": (lambda t: sg.sg_tile_cross_attention(p, two, two, two, two, run=t), torch.uint8, 2),
        "own_len": (lambda t: sg.sg_tile_prefix_attention(p, two, two, two, _Host(), _Host(), two, own_len=t), torch.int32, 2),
        "prefix_len": (lambda t: sg.sg_tile_prefix_attention(p, two, two, two, _Host(), _Host(), two, prefix_len=t), torch.int32, 1),
        "prefix_run": (lambda t: sg.sg_tile_prefix_attention(p, two, two, two, _Host(), _Host(), two, run=t), torch.uint8, 2),
        "norm_run": (lambda t: sg.sg_tile_residual_norm(n, two, None, two, run=t), torch.uint8, 2),
    }
    for name, (call, kind, size) in calls.items():
        for other in (torch.int64, torch.int32 if kind is torch.uint8 else torch.uint8, torch.float32, torch.int16):
            with pytest.raises(TypeError):
                call(_Device(torch.ones(size, dtype=other)))
        for wrong in (torch.ones(size - 1, dtype=kind), torch.ones(2 * size + 1, dtype=kind)[::2]):
            if wrong.is_contiguous() and wrong.numel() >= size:
                continue
            with pytest.raises(ValueError):
                call(_Device(wrong))
        with pytest.raises(ValueError):
            call(torch.ones(size, dtype=kind))   # on the host
    assert binding._flags(_Device(torch.ones(3, dtype=torch.bool)), 3, "run") and binding._lengths(None, 3, "own_len") is None
    longer = _Device(torch.ones(9, dtype=torch.int32))
    assert binding._lengths(longer, 3, "own_len") == longer.data_ptr()
