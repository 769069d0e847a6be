"""Outputs of context attention whose heads overlap are refused, at the largest strides and token counts too (host only)."""
import pytest

import paper_2508_17756_amd as sg

FAR = (1 << 40) - 8   # the largest stride


def _validate(heads, tokens, token, head):
    p = sg.make_context_problem(tokens, 20, heads, 64, "bf16")
    p.out_stride_token, p.out_stride_head = token, head
    return sg.sg_context_validate(p)


@pytest.mark.parametrize("heads, tokens, token, head, fits", [
    (2, 100, 64, 6400, True), (2, 100, 64, 6392, False), (2, 100, 72, 99 * 72 + 64, True), (2, 100, 72, 99 * 72 + 56, False),
    (5, 100, 320, 64, True), (5, 100, 312, 64, False), (5, 100, 4 * 72 + 64, 72, True), (5, 100, 4 * 72 + 56, 72, False),
    (5, 1, 64, 64, True), (5, 1, 64, 56, False), (1, 100, 64, 8, True),
    # (tokens - 1) * stride passes 2^63: head 1's token 0 is head 0's token 1
    (2, (1 << 24) - 1, FAR, FAR, False), (2, (1 << 24) - 1, FAR, FAR - 8, False), (2, (1 << 24) - 1, FAR, 64, True),
    ((1 << 24) - 1, 2, FAR, FAR, False), ((1 << 24) - 1, 2, 64, FAR, True), (2, (1 << 24) - 1, 64, ((1 << 24) - 1) * 64, True)])
def test_heads_of_an_output_do_not_overlap(heads, tokens, token, head, fits):
    want = sg.SG_ERR_INVALID_ARG if not fits else sg.SG_ERR_UNSUPPORTED if heads > 65535 else sg.SG_OK   # (65,535 heads of keys at most)
    assert _validate(heads, tokens, token, head) == want
