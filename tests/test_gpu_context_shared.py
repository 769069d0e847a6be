"""Context attention whose workgroups share stages of keys, and which kernels a call takes: places that do not count hold NaN, infinities or the
lowest values, results are compared with the formula in 64 bits, the largest difference and the mean square of all."""
import math
import re

import pytest
import torch

import paper_2508_17756_amd as sg
from context_util import U16, U32, Call

pytestmark = pytest.mark.gpu

CUS = 256   # the sizes below are chosen for this many compute units


@pytest.fixture(scope="module", autouse=True)
def _device():
    if torch.cuda.get_device_properties(0).multi_processor_count != CUS:
        pytest.skip("the sizes are those of a device with %d compute units" % CUS)


def kernels(call):
    """The context kernels that a call launches, with their template arguments (without those of the join)."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as trace:
        call()
        torch.cuda.synchronize()
    names = [e.key for e in trace.key_averages()]
    found = [re.search(r"context_(\w+)_kernel(?:<([^>]*)>)?", n) for n in names]
    found = [m.group(1) if m.group(1) == "join" else "%s<%s>" % (m.group(1), (m.group(2) or "").replace(" ", "")) for m in found if m]
    if not found and not any("sg::" in n for n in names):
        pytest.skip("no trace of kernels on this device")
    return sorted(found)


def _cross(tiles, tokens, heads, d, ctx, dtype="bf16", kv_heads=None, **kw):
    return lambda: Call(tiles, tokens, heads, kv_heads or heads, d, dtype, ctx, **kw)


def _prefix(tiles, tokens, heads, d, prefix, own, dtype="bf16", kv_heads=None, **kw):
    return lambda: Call(tiles, tokens, heads, kv_heads or heads, d, dtype, prefix, own=own, prefix=True, **kw)


# Either side of every rule of the cutting: bf16 <head_dim>, wide <head_dim, groups of wavefronts>, fp32 <head_dim, blocks of 16 rows, shared>
ROUTES = [
    ("token", _cross(1, 1, 8, 64, 77), ["bf16_split<64>"]),
    ("resident_from_4096_row_blocks", _cross(1, 2048, 64, 128, 256), ["bf16_resident<128>"]),
    ("below_4096_row_blocks", _cross(1, 2016, 64, 128, 256), ["bf16_wide<128,1>"]),
    ("more_keys_than_fit_128", _cross(1, 2048, 64, 128, 257), ["bf16_wide<128,1>"]),
    ("most_keys_that_fit_64", _cross(1, 2048, 64, 64, 512), ["bf16_resident<64>"]),
    ("more_keys_than_fit_64", _cross(1, 2048, 64, 64, 513), ["bf16_wide<64,1>"]),
    ("prefix_and_own_fit", _prefix(2, 1024, 64, 64, 200, 256), ["bf16_resident<64>"]),
    ("prefix_and_own_stages_do_not_fit", _prefix(2, 1024, 64, 64, 200, 257), ["bf16_wide<64,1>"]),
    ("shared_from_128_blocks", _cross(1, 1024, 16, 128, 77), ["bf16_wide<128,1>"]),
    ("below_128_blocks", _cross(1, 896, 16, 128, 77), ["bf16_split<128>"]),
    ("few_blocks_many_keys", _cross(1, 1024, 2, 128, 8000), ["bf16_wide<128,1>", "join"]),
    ("few_blocks_fewer_keys", _cross(1, 1024, 2, 128, 2000), ["bf16_split<128>", "join"]),
    ("two_groups", _cross(1, 1024, 32, 64, 512), ["bf16_wide<64,2>"]),
    ("two_groups_need_eight_stages", _cross(1, 1024, 32, 64, 448), ["bf16_wide<64,1>"]),
    ("two_groups_have_a_compute_unit_alone", _cross(1, 1024, 33, 64, 512), ["bf16_wide<64,1>"]),
    ("two_groups_cut", _cross(1, 1024, 4, 64, 8000), ["bf16_wide<64,2>", "join"]),
    ("stacked_shared", _prefix(20, 1, 40, 128, 2000, 40, kv_heads=8), ["bf16_split<128>", "bf16_wide<128,1>"]),
    ("stacked_shared_without_own_keys", _prefix(20, 1, 40, 128, 2000, 0, kv_heads=8), ["bf16_wide<128,1>", "join"]),
    ("stacked_shared_one_share", _prefix(20, 1, 40, 128, 700, 0, kv_heads=8), ["bf16_wide<128,1>"]),
    ("stacked_shared_own_keys_cut", _prefix(20, 4, 4, 128, 2000, 700, kv_heads=1), ["bf16_split<128>", "bf16_wide<128,1>", "join"]),
    ("too_many_rows_to_stack", _prefix(4, 17, 2, 128, 2000, 40), ["bf16_split<128>", "join"]),
    ("f32_token", _cross(1, 1, 8, 64, 77, "f32"), ["f32<64,1,false>"]),
    ("f32_shared_from_512_blocks", _cross(1, 2048, 16, 128, 77, "f32"), ["f32<128,1,true>"]),
    ("f32_below_512_blocks", _cross(1, 1984, 16, 128, 77, "f32"), ["f32<128,2,false>"]),
    ("f32_few_blocks_many_keys", _cross(2, 300, 8, 128, 1999, "f32"), ["f32<128,1,true>", "join"]),
    ("f32_shared_64", _cross(4, 520, 15, 64, 300, "f32"), ["f32<64,1,true>"]),
    ("f32_more_than_16_rows_64", _cross(1, 64, 2, 64, 16000, "f32"), ["f32<64,1,false>", "join"]),
    ("f32_32_rows_64", _cross(4, 440, 16, 64, 200, "f32"), ["f32<64,2,false>"]),
]


@pytest.mark.parametrize("name, make, want", ROUTES, ids=[r[0] for r in ROUTES])
def test_a_call_takes_its_kernels(name, make, want):
    assert kernels(make()) == want


SHARED = [
    ("wide_128", _cross(4, 600, 10, 128, 600), "bf16_wide<128,1>"),
    ("wide_128_token_major_grouped", _cross(4, 300, 20, 128, 600, kv_heads=10, lay="token"), "bf16_wide<128,1>"),
    ("wide_128_cut", _cross(4, 1000, 1, 128, 4100), "bf16_wide<128,1>"),
    ("wide_64", _cross(4, 700, 24, 64, 700, lay="odd"), "bf16_wide<64,1>"),
    ("two_groups", _cross(4, 500, 16, 64, 577), "bf16_wide<64,2>"),
    ("f32_128", _cross(4, 300, 26, 128, 150, "f32"), "f32<128,1,true>"),
    ("f32_128_cut", _cross(4, 300, 4, 128, 2001, "f32"), "f32<128,1,true>"),
    ("f32_64", _cross(4, 300, 52, 64, 300, "f32", kv_heads=26, lay="odd"), "f32<64,1,true>"),
]


def _dropped(c, i):
    drop = torch.ones(c.ctx, dtype=torch.bool)
    drop[c.keys(i)] = False
    return drop.to("cuda")


@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf"), -3.0e38])
@pytest.mark.parametrize("name, make, kernel", SHARED, ids=[s[0] for s in SHARED])
def test_what_does_not_count_is_not_seen_by_those_who_share(name, make, kernel, poison):
    """Whole stages and single places inside the length are masked, the last stage ends in the middle, one tile has no keys, one only masked ones."""
    c = make()
    n = c.ctx
    c.lens = torch.tensor([n - 1, 70, 0, n], dtype=torch.int32)
    c.mask = (torch.rand((4, n), generator=torch.Generator().manual_seed(5)) < 0.7).to(torch.uint8)
    c.mask[0, :128] = 0        # whole stages, the first ones
    c.mask[1, :70] = 0
    c.mask[3, 64:128] = 0
    c.mask[3, n - 30:] = 0
    clean = [[t.clone() for t in ts] for ts in (c.k, c.v)]
    for i in range(4):
        c.k[i][:, _dropped(c, i)] = poison
        c.v[i][:, _dropped(c, i)] = poison
    assert kernel in kernels(c)
    out = c()
    torch.cuda.synchronize()
    assert all(float(out[i].float().abs().max()) == 0 for i in (1, 2))
    c.k, c.v = clean
    c.check(out, heads=[0, c.heads - 1])


PREFIX_SHARED = [
    ("wide_128", _prefix(4, 600, 10, 128, 200, 333), "bf16_wide<128,1>"),
    ("two_groups", _prefix(4, 500, 16, 64, 200, 400), "bf16_wide<64,2>"),
    ("stacked", _prefix(4, 16, 8, 128, 900, 130, kv_heads=8), "bf16_split<128>"),
    ("stacked_shared", _prefix(20, 4, 8, 128, 900, 130), "bf16_wide<128,1>"),
    ("f32_128", _prefix(4, 300, 26, 128, 77, 140, "f32"), "f32<128,1,true>"),
]


@pytest.mark.parametrize("poison", [float("nan"), float("inf")])
@pytest.mark.parametrize("name, make, kernel", PREFIX_SHARED, ids=[s[0] for s in PREFIX_SHARED])
def test_behind_the_lengths_of_prefix_and_own_keys(name, make, kernel, poison):
    c = make()
    length = c.ctx - 70
    c.prefix_len = torch.tensor([length], dtype=torch.int32)
    c.lens = torch.tensor([c.own - 1, 0, 33, c.own] * (c.tiles // 4), dtype=torch.int32)
    clean = [[t.clone() for t in ts] for ts in (c.k, c.v)] + [c.pk.clone(), c.pv.clone()]
    for i in range(c.tiles):
        for t in (c.k[i], c.v[i]):
            t[:, int(c.lens[i]):] = poison
    c.pk[:, length:] = poison
    c.pv[:, length:] = poison
    assert kernel in kernels(c)
    out = c()
    torch.cuda.synchronize()
    c.k, c.v, c.pk, c.pv = clean
    c.check(out, heads=[0, c.heads - 1])


@pytest.mark.parametrize("name, make, kernel", SHARED, ids=[s[0] for s in SHARED])
def test_a_nan_that_counts_reaches_what_depends_on_it_through_shared_stages(name, make, kernel):
    c = make()
    group = c.heads // c.kv_heads
    c.q[0][c.heads - 1, 2, 5] = float("nan")
    c.v[1][0, c.ctx - 1, 3] = float("nan")
    c.k[2][0, 40, 7] = float("nan")
    out = c()
    torch.cuda.synchronize()
    for i in range(4):
        want = torch.zeros(out[i].shape, dtype=torch.bool)
        if i == 0:
            want[c.heads - 1, 2, :] = True
        elif i == 1:
            want[:group, :, 3] = True
        elif i == 2:
            want[:group] = True
        assert torch.equal(torch.isnan(out[i].cpu()), want), i


def rms_bound(d, keys, dtype):
    """Root of the mean square error over that of the results, for Q, K, V of N(0, 1) and scale d^-1/2.  A rounding's relative error has a mean square of
    at most 2^-48 / 3 (fp32).  A score, a chain of d products whose partial sums grow from 1 to d in mean square, gets (d^2 / 2 + d) / d times
    that, the scale 1 + 1 more, its exponent's argument (about 4 in size, two roundings, and what the reference's own may add) 2 x 16 x 2, the
    exponential 4; errors of different keys' probabilities are independent, so that the result has in proportion what one of them has.  The chain over the keys
    gets keys / 2 + 1, the sum of probabilities and the quotient keys / 2 + 2.  Twice the root, as errors are not quite independent.
    bf16: a probability and the result, 2^-16 / 3 at most each (the sum, of the rounded ones, makes it less)."""
    u2 = U32 * U32 / 3
    total = u2 * (d / 2 + 1 + 2 + 64 + 4 + keys / 2 + 1 + keys / 2 + 2)
    return 2 * math.sqrt(total) + (math.sqrt(2 * U16 * U16 / 3) if dtype == "bf16" else 0.0)


ACCURATE = [(name, make, kernel) for name, make, kernel in SHARED] + [
    ("f32_128_ragged", _cross(4, 300, 52, 128, 226, "f32", kv_heads=26, ragged=True, masked=True, run=True, lay="token"), "f32<128,1,true>"),
    ("f32_128_joint", _prefix(2, 650, 24, 128, 77, 650, "f32"), "f32<128,1,true>"),
    ("f32_128_split", _cross(4, 300, 4, 128, 300, "f32"), "f32<128,1,false>"),
    ("f32_64_split", _prefix(4, 300, 2, 64, 77, 300, "f32"), "f32<64,1,false>"),
    ("f32_32_rows", _cross(4, 440, 16, 64, 200, "f32"), "f32<64,2,false>"),
    ("f32_128_32_rows", _cross(1, 1984, 16, 128, 77, "f32"), "f32<128,2,false>"),
    ("bf16_split", _cross(2, 100, 8, 128, 300), "bf16_split<128>"),
    ("bf16_resident_128", _cross(1, 2048, 64, 128, 256), "bf16_resident<128>"),
    ("bf16_resident_64", _cross(1, 2048, 64, 64, 512), "bf16_resident<64>"),
    ("bf16_joint_64", _prefix(3, 650, 25, 64, 77, 650), "bf16_wide<64,1>"),
]


@pytest.mark.parametrize("name, make, kernel", ACCURATE, ids=[a[0] for a in ACCURATE])
def test_values_and_their_mean_square_error(name, make, kernel):
    c = make()
    before = [t.clone() for t in c.out]
    assert kernel in kernels(c)
    out = c()
    torch.cuda.synchronize()
    heads = [0, c.heads // 2, c.heads - 1]
    c.check(out, before, heads=heads)
    for i in range(c.tiles):
        n = len(c.keys(i)) + (c.ctx if c.prefix else 0)
        if n == 0 or (c.run is not None and int(c.run[i]) == 0):
            continue
        for a in heads:
            want, _ = c.reference(i, a)
            err = (out[i][a].cpu().double() - want).square().mean().sqrt() / want.square().mean().sqrt()
            assert float(err) <= rms_bound(c.d, n, c.dtype), "tile %d head %d: %.3e, bound %.3e" % (i, a, float(err), rms_bound(c.d, n, c.dtype))
