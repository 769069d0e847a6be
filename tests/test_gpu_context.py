"""Cross attention and shared-prefix attention of tiles against their formula in 64 bits, within the roundings the kernels make."""
import pytest
import torch

import paper_2508_17756_amd as sg
from context_util import Call

pytestmark = pytest.mark.gpu

DT = ["bf16", "f32"]


def _run(c, **kw):
    before = [t.clone() for t in c.out]
    out = c(**kw)
    torch.cuda.synchronize()
    c.check(out, before)
    return out


# tokens (queries), context lengths around the stages of 16, 32 and 64 keys, and around the blocks of 16, 32 and 128 queries
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens, ctx", [(1, 1), (1, 0), (1, 77), (2, 15), (3, 16), (5, 17), (16, 31), (17, 32), (31, 33), (32, 63), (33, 64),
                                         (63, 65), (100, 226), (129, 127), (128, 128), (257, 129), (300, 300)])
def test_cross_sizes(dtype, d, tokens, ctx):
    _run(Call(2, tokens, 3, 3, d, dtype, ctx, seed=tokens + ctx))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("d, heads, kv_heads", [(64, 4, 1), (128, 4, 2), (128, 6, 2), (64, 10, 5), (128, 40, 8)])
@pytest.mark.parametrize("lay", ["packed", "token", "odd"])
def test_cross_grouped_heads_and_strides(dtype, d, heads, kv_heads, lay):
    _run(Call(3, 21, heads, kv_heads, d, dtype, 90, lay=lay, ragged=True, masked=True, run=True, seed=heads))


# enough rows for the kernel whose workgroups share their keys (256 workgroups of 128 rows), and a few less
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lay", ["packed", "token", "odd"])
@pytest.mark.parametrize("tiles, tokens, heads, kv_heads, ctx", [(2, 1000, 17, 17, 77), (4, 129, 32, 32, 130), (3, 700, 16, 16, 64),
                                                                  (2, 500, 64, 32, 200), (2, 1000, 15, 15, 77)])
def test_cross_many_rows(d, lay, tiles, tokens, heads, kv_heads, ctx):
    c = Call(tiles, tokens, heads, kv_heads, d, "bf16", ctx, lay=lay, ragged=True, masked=True, run=tiles > 2, seed=ctx)
    before = [t.clone() for t in c.out]
    c()
    torch.cuda.synchronize()
    c.check(c.out, before, heads=[0, 1, heads // 2, heads - 1])


# more row blocks than the wavefronts that keep a head's keys in LDS take at once (two for each of 256 x 8): the most keys that fit, one, none;
# grouped heads, ranges of row blocks that pass from head to head and from tile to tile
@pytest.mark.parametrize("lay", ["packed", "token", "odd"])
@pytest.mark.parametrize("d, tiles, tokens, heads, kv_heads, ctx", [(64, 4, 540, 64, 64, 512), (128, 4, 540, 64, 64, 256), (64, 3, 2100, 24, 24, 226),
                                                                    (128, 3, 2100, 24, 24, 77), (64, 5, 300, 128, 32, 130), (64, 65, 33, 64, 32, 40),
                                                                    (128, 2, 33, 1024, 1024, 1)])
def test_cross_over_few_keys(lay, d, tiles, tokens, heads, kv_heads, ctx):
    c = Call(tiles, tokens, heads, kv_heads, d, "bf16", ctx, lay=lay, ragged=True, masked=ctx > 1, run=tiles > 2, seed=ctx)
    before = [t.clone() for t in c.out]
    c()
    torch.cuda.synchronize()
    c.check(c.out, before, heads=[0, 1, heads // 2, heads - 1])


@pytest.mark.parametrize("lay", ["packed", "odd"])
@pytest.mark.parametrize("d, own, prefix", [(64, 130, 300), (128, 60, 190), (64, 1, 1), (64, 0, 512), (128, 256, 0)])
def test_prefix_and_own_keys_that_fit(lay, d, own, prefix):
    for length in (None, 0, prefix // 2):
        c = Call(4, 540, 64, 64, d, "bf16", prefix, own=own, prefix=True, lay=lay, ragged=own > 0, run=True, seed=own)
        c.prefix_len = None if length is None else torch.tensor([length], dtype=torch.int32)
        before = [t.clone() for t in c.out]
        c()
        torch.cuda.synchronize()
        c.check(c.out, before, heads=[0, 31, 63])


# few blocks of 128 rows over many keys, shared and cut into shares, which a second launch joins
@pytest.mark.parametrize("dtype, d, tiles, tokens, heads, kv_heads, ctx", [
    ("bf16", 128, 1, 1000, 2, 2, 8000), ("bf16", 64, 2, 500, 16, 8, 2001), ("bf16", 128, 3, 129, 8, 4, 1500), ("f32", 128, 2, 300, 8, 8, 1999),
    ("f32", 64, 1, 600, 16, 16, 2500), ("bf16", 64, 3, 400, 25, 25, 1031), ("bf16", 64, 1, 1000, 8, 4, 8003)])
@pytest.mark.parametrize("lay", ["packed", "odd"])
def test_cross_of_many_rows_and_keys(dtype, d, tiles, tokens, heads, kv_heads, ctx, lay):
    for prefix in (False, True):
        c = Call(tiles, tokens, heads, kv_heads, d, dtype, 500 if prefix else ctx, own=ctx - 500 if prefix else 0, prefix=prefix, lay=lay,
                 ragged=tiles > 1, masked=not prefix, run=tiles > 2, seed=ctx)
        before = [t.clone() for t in c.out]
        c()
        torch.cuda.synchronize()
        c.check(c.out, before, heads=[0, heads - 1])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tiles, tokens, heads, kv_heads, own, prefix", [
    (1, 1, 2, 2, 1, 1), (3, 1, 8, 2, 40, 200), (20, 1, 4, 4, 3, 1000), (5, 4, 8, 2, 33, 513), (2, 16, 3, 3, 16, 129), (4, 17, 4, 2, 17, 300),
    (2, 100, 3, 3, 100, 77), (1, 200, 4, 4, 200, 64), (3, 1, 4, 4, 0, 300), (3, 2, 4, 4, 300, 0), (2, 1, 2, 2, 0, 0), (2, 40, 2, 2, 0, 50)])
def test_prefix_sizes(dtype, d, tiles, tokens, heads, kv_heads, own, prefix):
    _run(Call(tiles, tokens, heads, kv_heads, d, dtype, prefix, own=own, prefix=True, ragged=own > 0, seed=own + prefix))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tiles, tokens, heads, kv_heads, own, prefix", [
    (20, 1, 10, 2, 0, 130), (20, 1, 10, 2, 31, 1300), (33, 4, 2, 1, 0, 900), (40, 1, 16, 4, 700, 2000), (17, 8, 2, 1, 64, 128), (64, 16, 1, 1, 5, 640),
    (13, 5, 6, 6, 2000, 700)])
def test_prefix_of_more_stacked_rows_than_a_wavefront_takes(dtype, d, tiles, tokens, heads, kv_heads, own, prefix):
    for length in (None, prefix // 3):
        c = Call(tiles, tokens, heads, kv_heads, d, dtype, prefix, own=own, prefix=True, lay="token", ragged=own > 0, run=True, seed=own + prefix)
        c.prefix_len = None if length is None else torch.tensor([length], dtype=torch.int32)
        _run(c)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("lay", ["packed", "token", "odd"])
@pytest.mark.parametrize("tokens", [1, 30])
def test_prefix_strides_lengths_and_skipped_tiles(dtype, lay, tokens):
    for length in (None, 0, 1, 150, 10**9, -5):
        c = Call(5, tokens, 6, 2, 128, dtype, 260, own=70, prefix=True, lay=lay, ragged=True, run=True, seed=tokens)
        c.prefix_len = None if length is None else torch.tensor([length], dtype=torch.int32)
        _run(c)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lay", ["packed", "token", "odd"])
def test_prefix_many_rows(d, lay):
    """Joint attention of text and tile with rows to fill the chip; the text ends inside a stage, and so do the tiles."""
    c = Call(3, 650, 16, 16, d, "bf16", 77, own=650, prefix=True, lay=lay, ragged=True, run=True, seed=d)
    before = [t.clone() for t in c.out]
    c()
    torch.cuda.synchronize()
    c.check(c.out, before, heads=[0, 7, 15])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("tokens", [1, 300])
def test_lengths_outside_the_buffers_are_clamped(dtype, tokens):
    c = Call(4, tokens, 16, 16, 64, dtype, 50, ragged=True)
    c.lens = torch.tensor([-3, 10**6, 2**31 - 1, -2**31], dtype=torch.int32)
    c()
    c.lens = torch.tensor([0, 50, 50, 0], dtype=torch.int32)
    c.check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("tokens, heads", [(1, 4), (40, 4), (600, 64)])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -3.0e38])
def test_what_does_not_count_is_not_read(dtype, tokens, heads, poison):
    """Masked places and places behind the length hold NaN, infinities or the lowest values: the result is that of the others alone."""
    c = Call(2, tokens, heads, heads, 64 if heads > 4 else 128, dtype, 150, ragged=True, masked=True, seed=3)
    c.lens = torch.tensor([149, 70], dtype=torch.int32)
    c.mask = (torch.rand((2, 150), generator=torch.Generator().manual_seed(5)) < 0.6).to(torch.uint8)
    c.mask[1, 64:] = 0
    c.mask[0, :64] = 0   # a whole stage
    clean = [[t.clone() for t in ts] for ts in (c.k, c.v)]
    for i in range(2):
        drop = torch.ones(150, dtype=torch.bool)
        drop[c.keys(i)] = False
        c.k[i][:, drop.to("cuda")] = poison
        c.v[i][:, drop.to("cuda")] = poison
    out = [t.clone() for t in c()]
    c.k, c.v = clean
    c.check(out, heads=range(4))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("tokens, heads", [(3, 2), (600, 64)])
def test_a_nan_reaches_what_depends_on_it_and_nothing_else(dtype, tokens, heads):
    c = Call(2, tokens, heads, heads, 128, dtype, 100, seed=9)
    c.q[0][1, 2, 5] = float("nan")       # one query
    c.v[1][0, 70, 3] = float("nan")      # one channel of a head of the second tile
    out = c()
    torch.cuda.synchronize()
    for i in range(2):
        want = torch.zeros(out[i].shape, dtype=torch.bool)
        if i == 0:
            want[1, 2, :] = True
        else:
            want[0, :, 3] = True
        assert torch.equal(torch.isnan(out[i].cpu()), want)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("tokens, heads, spread", [(5, 2, 8.0), (400, 90, 8.0), (5, 2, 30.0)])
def test_peaked_softmax_and_rising_maxima(dtype, tokens, heads, spread):
    """Scores of up to thousands, rising along the keys: the reference moves at every stage."""
    c = Call(1, tokens, heads, heads, 64, dtype, 500, spread=spread, seed=11)
    ramp = torch.linspace(0.05, 1.0, 500, device="cuda").to(c.k[0].dtype)
    c.k[0] *= ramp[None, :, None]
    c()
    torch.cuda.synchronize()
    c.check(heads=[0, heads - 1])


def test_constant_scores_and_large_values():
    """K = 0: the mean of V; |V| near the largest number: finite."""
    for dtype, big in (("bf16", 3.0e38), ("f32", 1.0e38)):
        for tokens, heads in ((1, 2), (600, 64)):
            c = Call(1, tokens, heads, heads, 128, dtype, 90)
            c.k[0].zero_()
            c.v[0].fill_(big / 128)
            out = c()[0].float()
            want = float(c.v[0][0, 0, 0].float())
            assert bool(torch.isfinite(out).all()) and float((out / want - 1).abs().max()) < 2.0 ** -8 + 200 * 2.0 ** -24


@pytest.mark.parametrize("tiles", [64, 65, 130])
def test_more_tiles_than_a_launch_takes(tiles):
    for prefix in (False, True):
        c = Call(tiles, 2, 2, 1, 64, "bf16", 300, own=20, prefix=prefix, ragged=True, masked=not prefix, run=True, seed=tiles)
        _run(c)


def test_many_tiles_of_many_rows():
    c = Call(70, 140, 4, 4, 64, "bf16", 33, ragged=True, masked=True, run=True, seed=1)
    before = [t.clone() for t in c.out]
    c()
    torch.cuda.synchronize()
    c.check(c.out, before, heads=[0, 3])


@pytest.mark.parametrize("dtype", DT)
def test_a_long_prefix_whose_offsets_pass_32_bits(dtype):
    """The last keys of the prefix lie beyond 4 GiB of its first."""
    heads, d, n, token = 2, 128, 1200, 1 << 21   # 1,200 keys, 2^21 elements apart
    c = Call(3, 2, heads, heads, d, dtype, n, own=10, prefix=True, seed=2)
    for name in ("pk", "pv"):
        packed = getattr(c, name)
        flat = torch.zeros((n - 1) * token + heads * d, dtype=packed.dtype, device="cuda")
        assert (n - 1) * token * flat.element_size() > 1 << 32
        spread = flat.as_strided((heads, n, d), (d, token, 1))
        spread.copy_(packed)
        setattr(c, name, spread)
    c.p.ctx_stride_token, c.p.ctx_stride_head = token, d
    c()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("tiles, tokens, heads, own, prefix", [(4, 1, 8, 40, 900), (2, 600, 64, 0, 50)])
def test_replays_from_a_graph(dtype, tiles, tokens, heads, own, prefix):
    """Captured and replayed with eager work in between; lengths and inputs change in place, and a second graph shares the workspace on
    the same stream."""
    c = Call(tiles, tokens, heads, heads, 64, dtype, prefix, own=own, prefix=True, seed=4)
    lens = torch.full((1,), prefix, dtype=torch.int32, device="cuda")
    ws = c.workspace()
    eager, graphed = [torch.zeros_like(t) for t in c.out], [torch.zeros_like(t) for t in c.out]

    def call(out):
        sg.sg_tile_prefix_attention(c.p, c.q, c.k if own else None, c.v if own else None, c.pk, c.pv, out, prefix_len=lens, workspace=ws)

    call(eager)
    torch.cuda.synchronize()
    graphs, side = [], torch.cuda.Stream()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            call(graphed)
        graphs.append(g)
    torch.cuda.synchronize()
    for k in range(4):
        lens.fill_(max(1, prefix - 13 * k))
        c.pv.mul_(0.75)
        call(eager)
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        for x, y in zip(eager, graphed):
            assert torch.equal(x, y)
    c.prefix_len = lens
    c.check(graphed, heads=[0, heads - 1])


def test_streams_and_repeats_give_the_same_bits():
    """Two calls at once on two streams, a workspace each; and the same call again."""
    c = Call(6, 1, 16, 4, 128, "bf16", 2000, own=100, prefix=True, ragged=True, seed=8)
    want = [t.clone() for t in c()]
    torch.cuda.synchronize()
    outs = [[torch.zeros_like(t) for t in c.out] for _ in range(2)]
    spaces = [c.workspace() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, ws in zip(streams, outs, spaces):
            with torch.cuda.stream(s):
                c(workspace=ws, out=o)
    torch.cuda.synchronize()
    for o in outs:
        for x, y in zip(o, want):
            assert torch.equal(x, y)


def test_a_dirty_workspace_and_outputs_beside_the_rows():
    """Nothing but the rows is written, whatever the workspace holds."""
    for dtype in DT:
        for tokens, heads in ((1, 6), (50, 6), (500, 70)):
            c = Call(2, tokens, heads, heads, 64, dtype, 400, lay="odd", seed=tokens)
            ws = c.workspace()
            ws.fill_(255)
            stores = [t.as_strided((heads * c.p.out_stride_head,), (1,)) for t in c.out]
            for t in stores:
                t.fill_(7.0)
            c(workspace=ws)
            torch.cuda.synchronize()
            c.check(heads=[0, heads - 1])
            for t, o in zip(stores, c.out):
                o.fill_(7.0)
                assert bool((t == 7.0).all())


def test_refused_on_the_device_side_too():
    c = Call(2, 1, 8, 8, 128, "bf16", 30000, own=8, prefix=True)
    with pytest.raises(sg.SgError):
        sg.sg_tile_prefix_attention(c.p, c.q, c.k, c.v, c.pk, c.pv, c.out)      # no workspace
    with pytest.raises(sg.SgError):
        sg.sg_tile_prefix_attention(c.p, c.q, c.k, c.v, c.pk, None, c.out, workspace=c.workspace())


@pytest.mark.parametrize("d, ctx", [(64, 500), (128, 250)])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -3.0e38])
def test_what_does_not_count_is_not_read_into_lds(d, ctx, poison):
    c = Call(4, 540, 64, 64, d, "bf16", ctx, ragged=True, masked=True, seed=3)
    c.lens = torch.tensor([ctx - 1, 70, 0, ctx], dtype=torch.int32)
    c.mask[0, :64] = 0
    clean = [[t.clone() for t in ts] for ts in (c.k, c.v)]
    for i in range(4):
        drop = torch.ones(ctx, dtype=torch.bool)
        drop[c.keys(i)] = False
        c.k[i][:, drop.to("cuda")] = poison
        c.v[i][:, drop.to("cuda")] = poison
    out = [t.clone() for t in c()]
    c.k, c.v = clean
    c.check(out, heads=[0, 33])
    # a NaN that counts, in one channel of a head of the first tile
    at = int(c.keys(0)[5])
    c.v[0][7, at, 3] = float("nan")
    c.q[1][9, 11, 0] = float("nan")
    out = c()
    torch.cuda.synchronize()
    for i in range(4):
        want = torch.zeros(out[i].shape, dtype=torch.bool)
        if i == 0:
            want[7, :, 3] = True
        if i == 1:
            want[9, 11, :] = True
        assert torch.equal(torch.isnan(out[i].cpu()), want)


@pytest.mark.parametrize("d, ctx", [(64, 512), (128, 256)])
def test_rising_maxima_over_few_keys(d, ctx):
    c = Call(1, 2100, 64, 64, d, "bf16", ctx, spread=8.0, seed=11)
    c.k[0] *= torch.linspace(0.05, 1.0, ctx, device="cuda").to(c.k[0].dtype)[None, :, None]
    c()
    torch.cuda.synchronize()
    c.check(heads=[0, 63])


@pytest.mark.parametrize("tokens, heads, ctx", [(2100, 64, 300), (1000, 2, 6000)])
def test_replays_of_cross_attention_with_changing_flags(tokens, heads, ctx):
    """Lengths, masks and run flags are read by every replay; rows of a tile that does not run stay."""
    c = Call(2, tokens, heads, heads, 64, "bf16", ctx, seed=6)
    lens = torch.full((2,), ctx, dtype=torch.int32, device="cuda")
    mask = torch.ones((2, ctx), dtype=torch.uint8, device="cuda")
    run = torch.ones((2,), dtype=torch.uint8, device="cuda")
    ws = c.workspace()
    eager, graphed = [torch.zeros_like(t) for t in c.out], [torch.zeros_like(t) for t in c.out]

    def call(out):
        sg.sg_tile_cross_attention(c.p, c.q, c.k, c.v, out, ctx_len=lens, key_mask=mask, run=run, workspace=ws)

    call(eager)
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        call(graphed)
    torch.cuda.synchronize()
    g.replay()
    for k in range(4):
        lens.copy_(torch.tensor([ctx - 31 * k, 100 * k], dtype=torch.int32))
        mask[:, k::7] = 0
        run[k & 1] = k < 2
        c.q[0].mul_(0.9)
        call(eager)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager, graphed):
            assert torch.equal(x, y)


def test_two_calls_at_once_of_every_kind():
    """Calls of different shapes on two streams, a workspace each, give what they give alone."""
    calls = [Call(4, 540, 64, 64, 64, "bf16", 300, seed=1), Call(1, 1000, 4, 4, 128, "bf16", 4000, seed=2),
             Call(20, 1, 8, 2, 128, "bf16", 3000, own=40, prefix=True, seed=3), Call(2, 300, 8, 8, 128, "f32", 1500, seed=4)]
    want = [[t.clone() for t in c()] for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[[torch.zeros_like(t) for t in c.out] for c in calls] for _ in streams]
    spaces = [[c.workspace() for c in calls] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for turn in range(len(calls)):
            for i, s in enumerate(streams):
                at = (turn + i) % len(calls)
                with torch.cuda.stream(s):
                    calls[at](workspace=spaces[i][at], out=got[i][at])
    torch.cuda.synchronize()
    for outs in got:
        for o, w in zip(outs, want):
            for x, y in zip(o, w):
                assert torch.equal(x, y)


def test_the_same_buffers_for_every_tile():
    """Tiles may name the same context, and the same queries."""
    c = Call(5, 40, 8, 2, 128, "bf16", 200, ragged=True, seed=5)
    c.q, c.k, c.v = [c.q[0]] * 5, [c.k[0]] * 5, [c.v[0]] * 5
    c.lens = torch.tensor([200, 0, 3, 64, 65], dtype=torch.int32)
    _run(c)


@pytest.mark.parametrize("lens", [[577, 0, 1, 64], [65, 128, 129, 1]])
def test_two_groups_of_a_workgroup_with_unequal_shares(lens):
    """Tiles whose keys fill no stage, one, an odd number of them: one group of wavefronts may have nothing."""
    c = Call(4, 500, 16, 16, 64, "bf16", 577, masked=True, seed=2)
    c.lens = torch.tensor(lens, dtype=torch.int32)
    c.mask[0, :512] = 0
    c.mask[3] = 1
    c()
    torch.cuda.synchronize()
    c.check(heads=[0, 15])
