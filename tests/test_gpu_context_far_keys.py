"""Context attention, keys far below the largest score: fp32 probabilities below 2^-126 count, in every kernel and in every join; scores at -inf have
probability 0."""
import pytest
import torch

from context_util import Call

pytestmark = pytest.mark.gpu


def _cross(tiles, tokens, heads, d, ctx, dtype="f32"):
    return lambda: Call(tiles, tokens, heads, heads, d, dtype, ctx)


def _prefix(tiles, tokens, heads, kv_heads, d, prefix, own, dtype="f32"):
    return lambda: Call(tiles, tokens, heads, kv_heads, d, dtype, prefix, own=own, prefix=True)


# as many rows as 16 or 32 to a wavefront, as workgroups that share their keys take; keys cut inside a workgroup, over workgroups, over launches
CALLS = [("token", _cross(1, 1, 8, 64, 77)), ("16_rows", _prefix(4, 300, 2, 2, 64, 77, 300)), ("32_rows_64", _cross(4, 440, 16, 64, 200)),
         ("32_rows_128", _cross(1, 1984, 16, 128, 77)), ("shared_128", _cross(4, 300, 26, 128, 150)), ("shared_64", _cross(4, 520, 15, 64, 300)),
         ("shared_cut", _cross(2, 300, 8, 128, 1999)), ("16_rows_joined", _cross(1, 64, 2, 64, 16000)), ("stacked", _prefix(20, 1, 8, 8, 128, 900, 130)),
         ("stacked_shared", _prefix(20, 4, 4, 4, 128, 2000, 70)), ("stacked_cut", _prefix(3, 1, 4, 2, 128, 1000, 900))]


def _constant(c, far, large):
    """Scores of 0 (so that the sum of probabilities is the number of keys) and of -90 for the keys `far` of prefix and own keys behind one another;
    values of 0, and `large` there.  q * scale is 1 and every product exact."""
    c.p.scale = 0.125
    for q in c.q:
        q.zero_()
        q[..., 0] = 8.0
    n0 = c.ctx if c.prefix else 0
    for kv, base in [((c.k[i], c.v[i]), n0) for i in range(c.tiles)] + ([((c.pk, c.pv), 0)] if c.prefix else []):
        for t in kv:
            t.zero_()
        for m in far:
            if 0 <= m - base < kv[0].shape[1]:
                kv[0][:, m - base, 0] = -90.0
                kv[1][:, m - base] = large
    return (c.own + n0) if c.prefix else c.ctx


@pytest.mark.parametrize("name, make", CALLS, ids=[c[0] for c in CALLS])
def test_a_key_far_below_the_largest_score_counts(name, make):
    """e^-90 = 8e-40 times 3e38 is 0.25.  The probability has 20 bits, 2^-20; its exponent, 129.84, is off by half of 2^-16 and by 2^-25 of itself from
    log2(e), times ln 2 together 8e-6; sums of n terms n 2^-24."""
    for where in ("first", "middle", "last"):
        c = make()
        n = c.own + c.ctx if c.prefix else c.ctx
        at = {"first": 0, "middle": n // 2, "last": n - 1}[where]
        _constant(c, [at], 3e38)
        out = c()
        torch.cuda.synchronize()
        large = float(torch.tensor(3e38, dtype=torch.float32))
        p = float(torch.tensor(-90.0, dtype=torch.float64).exp())
        want = p * large / (n - 1 + p)
        for o in out:
            assert float((o.double() / want - 1).abs().max()) <= 2.0 ** -20 + 8.1e-6 + (n + 64) * 2.0 ** -24, where


@pytest.mark.parametrize("name, make", CALLS, ids=[c[0] for c in CALLS])
def test_scores_near_the_largest_number(name, make):
    """All scores 3e38, one of them 2.9e38 (its probability is 0): the mean of the others' values, 1."""
    c = make()
    n = _constant(c, [0], 5.0)
    big, less = 3e38, 2.9e38
    for t in c.k + ([c.pk] if c.prefix else []):
        t[..., 0] = torch.where(t[..., 0] == 0, big, less)
    for t in c.v + ([c.pv] if c.prefix else []):
        t[:] = torch.where(t == 0, 1.0, 5.0)
    out = c()
    torch.cuda.synchronize()
    for o in out:
        assert float((o - 1).abs().max()) <= (n + 64) * 2.0 ** -24


BF16_CALLS = [("bf16_token", _cross(1, 1, 8, 64, 77, "bf16")), ("bf16_split", _cross(2, 100, 8, 128, 300, "bf16")),
              ("bf16_split_joined", _cross(1, 1024, 2, 128, 2000, "bf16")), ("bf16_wide_128", _cross(4, 600, 10, 128, 600, "bf16")),
              ("bf16_wide_64", _cross(4, 700, 24, 64, 700, "bf16")), ("bf16_wide_cut", _cross(1, 1024, 2, 128, 8000, "bf16")),
              ("bf16_two_groups", _cross(1, 1024, 32, 64, 512, "bf16")), ("bf16_resident_64", _cross(1, 2048, 64, 64, 512, "bf16")),
              ("bf16_resident_128", _cross(1, 2048, 64, 128, 256, "bf16")), ("bf16_stacked", _prefix(20, 1, 40, 8, 128, 2000, 40, "bf16")),
              ("bf16_stacked_cut", _prefix(20, 4, 4, 1, 128, 2000, 700, "bf16"))]


@pytest.mark.parametrize("name, make", CALLS + BF16_CALLS, ids=[c[0] for c in CALLS + BF16_CALLS])
def test_scores_at_minus_infinity(name, make):
    """Every head's first keys, its last ones, all but one, and all of them (zeros)."""
    inf = float("inf")
    for which in ("first", "last", "all_but_one", "all"):
        c = make()
        c.p.scale = 0.125
        n0 = c.ctx if c.prefix else 0
        n = c.own + n0 if c.prefix else c.ctx
        left = {"first": range(n // 2, n), "last": range(0, max(1, n // 3)), "all_but_one": range(n // 2, n // 2 + 1), "all": range(0)}[which]
        for q in c.q:
            q.zero_()
            q[..., 0] = 8.0
        lists = [((c.k[i], c.v[i]), n0) for i in range(c.tiles)] + ([((c.pk, c.pv), 0)] if c.prefix else [])
        for (k, v), base in lists:
            at = torch.arange(k.shape[1], device="cuda") + base
            k.zero_()
            k[..., 0] = torch.where((at >= left.start) & (at < left.stop), 0.0, -inf).to(k.dtype)
            v[:] = (at % 5 + 1)[:, None].to(v.dtype)
        out = c()
        torch.cuda.synchronize()
        want = 0.0 if which == "all" else sum(m % 5 + 1 for m in left) / len(left)
        step = 2.0 ** -8 if c.dtype == "bf16" else 2.0 ** -24
        for o in out:
            assert float((o.double() - want).abs().max()) <= (step + (n + 64) * 2.0 ** -24) * want, which
