"""Rotary positions of tiles against the formula in 64 bits, within the roundings the kernel makes."""
import pytest
import torch

import paper_2508_17756_amd as sg
from block_util import TORCH, check, rotary64, same

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, size=(2, 5, 7), heads=3, d=64, axes=(20, 22, 22), dtype="bf16", kv_heads=None, layout="interleaved", tiles=2, token_major=False,
                 wrap=None, origin=None, listed=0, columns=1, norm=False, pad=0, keys=True, seed=0, gain=1.0, **scaling):
        self.g = torch.Generator().manual_seed(400 + seed)
        self.size, self.heads, self.kv, self.d, self.axes, self.dtype = size, heads, kv_heads or heads, d, axes, dtype
        self.layout, self.tiles, self.token_major, self.wrap, self.keys = layout, tiles, token_major, wrap, keys
        n = self.n = size[0] * size[1] * size[2]
        self.p = sg.make_rotary_problem(size, heads, d, dtype, axes, kv_heads=kv_heads, layout=layout, wrap=wrap, position_axes=columns,
                                        token_major=token_major)
        if pad:
            for name, a in (("q", heads), ("q_out", heads), ("k", self.kv), ("k_out", self.kv)):
                setattr(self.p, name + "_stride_token", (a * d if token_major else d) + pad)
                setattr(self.p, name + "_stride_head", d if token_major else n * (d + pad) + pad)
        self.freq = sg.sg_rotary_frequencies(self.p, **scaling)
        self.q, self.k = ([self._new(a, gain) for _ in range(tiles)] for a in (heads, self.kv))
        self.q_out, self.k_out = ([torch.full_like(t, 7.0) for t in ts] for ts in (self.q, self.k))
        self.wq, self.wk = ((1 + 0.2 * torch.randn(d, generator=self.g)).to(TORCH[dtype]).cuda() if norm else None for _ in range(2))
        self.origin = self.positions = None
        if listed:
            self.positions = [torch.randint(-listed, listed, (n, columns), generator=self.g, dtype=torch.int32).cuda() for _ in range(tiles)]
        else:
            self.origin = origin or [(0, 3 * i, 50 * i + 1) for i in range(tiles)]

    def _new(self, a, gain):
        shape = self.flat(a)
        return (gain * torch.randn(shape, generator=self.g)).to(TORCH[self.dtype]).cuda()

    def flat(self, a):
        name = "q" if a == self.heads else "k"
        st, sh = getattr(self.p, name + "_stride_token"), getattr(self.p, name + "_stride_head")
        return (self.n - 1) * st + (a - 1) * sh + self.d

    def view(self, t, key):
        a = self.heads if key == "q" else self.kv
        return t.as_strided((self.n, a, self.d), (getattr(self.p, key + "_stride_token"), getattr(self.p, key + "_stride_head"), 1))

    def run(self, **kw):
        args = dict(origin=self.origin, positions=self.positions, q_weight=self.wq, k_weight=self.wk)
        if self.keys:
            args.update(k=self.k, k_out=self.k_out)
        sg.sg_tile_rotary(self.p, self.q, self.q_out, self.freq, **{**args, **kw})
        torch.cuda.synchronize()
        return self

    def coords(self, i):
        if self.positions is not None:
            return self.positions[i].cpu().expand(-1, 3)
        at = torch.arange(self.n)
        _, h, w = self.size
        c = torch.stack([at // (h * w), at // w % h, at % w], dim=1) + torch.tensor(self.origin[i])
        return c if self.wrap is None else torch.stack([c[:, j] % self.wrap[j] if self.wrap[j] else c[:, j] for j in range(3)], dim=1)

    def check(self, tiles=None):
        for i in range(self.tiles) if tiles is None else tiles:
            for key, xs, ys, w in (("q", self.q, self.q_out, self.wq), ("k", self.k, self.k_out, self.wk))[:2 if self.keys else 1]:
                ref, tol = rotary64(self.view(xs[i], key).cpu(), self.freq.cpu(), self.coords(i), self.axes, self.layout, None if w is None else w.cpu())
                check(self.view(ys[i], key), ref, tol, self.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("heads, kv_heads, d, axes", [
    (3, 3, 64, (20, 22, 22)), (5, 1, 128, (44, 42, 42)), (1, 1, 32, (4, 6, 6)), (2, 4, 96, (0, 48, 48)), (8, 2, 128, (128, 0, 0)),
    (40, 8, 128, (16, 0, 16)), (1, 1, 256, (2, 2, 12)), (2, 1, 512, (256, 128, 128)), (3, 1, 80, (0, 0, 32)), (1, 2, 16, (16, 0, 0)), (7, 7, 24, (2, 4, 10))])
@pytest.mark.parametrize("norm", [False, True])
def test_heads_and_axes(dtype, layout, heads, kv_heads, d, axes, norm):
    Call(heads=heads, kv_heads=kv_heads, d=d, axes=axes, dtype=dtype, layout=layout, norm=norm).run().check()
    Call(heads=heads, kv_heads=kv_heads, d=d, axes=axes, dtype=dtype, layout=layout, norm=norm, token_major=True, size=(1, 3, 11), tiles=1).run().check()


@pytest.mark.parametrize("d, axes", [(8, (2, 0, 0)), (8, (0, 4, 4)), (64, (2, 4, 4)), (40, (6, 6, 6)), (128, (0, 0, 126)), (72, (10, 10, 10))])
def test_interleaved_turns_any_even_number_of_channels(d, axes):
    Call(d=d, axes=axes, heads=4).run().check()
    Call(d=d, axes=axes, heads=4, dtype="f32", norm=True).run().check()


@pytest.mark.parametrize("size", [(1, 1, 1), (1, 1, 2), (2, 1, 1), (1, 9, 1), (3, 8, 8), (1, 1, 65), (5, 13, 17), (1, 64, 64)])
@pytest.mark.parametrize("heads", [1, 12])
def test_sizes(size, heads):
    Call(size=size, heads=heads, d=128, axes=(44, 42, 42), token_major=True, norm=True).run().check()
    Call(size=size, heads=heads, d=64, axes=(16, 8, 8), layout="half", keys=False).run().check()
    Call(size=size, heads=heads, kv_heads=1, d=64, axes=(16, 8, 8), layout="half", tiles=20).run().check()


@pytest.mark.parametrize("columns", [1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_listed_positions(dtype, columns):
    """Positions of millions, negative ones among them: fp32 angles would be off by a tenth of a turn."""
    Call(size=(33, 1, 1), heads=8, kv_heads=2, d=128, axes=(64, 32, 32), dtype=dtype, listed=1 << 23, columns=columns, layout="half").run().check()
    Call(size=(1, 1, 1), heads=40, kv_heads=8, d=128, axes=(128, 0, 0), dtype=dtype, listed=1 << 20, columns=columns, tiles=20, token_major=True).run().check()


@pytest.mark.parametrize("wrap", [(2, 9, 12), (0, 9, 12), (2, 0, 0), (1, 5, 3)])
def test_positions_wrap_around_the_canvas(wrap):
    Call(wrap=wrap, origin=[(0, 8, 11), (1, 100, 25)], dtype="f32").run().check()
    Call(wrap=wrap, origin=[(-3, -8, -1), (5, -2000000000, 2000000000 if wrap[2] else 7)], dtype="f32").run().check()


def test_a_wrapped_tile_meets_the_tokens_of_the_other_edge():
    """The same tokens at the same canvas places get the same bits, whatever tile they are in."""
    size, canvas = (1, 4, 6), (1, 8, 10)
    c = Call(size=size, wrap=canvas, origin=[(0, 6, 8), (0, 0, 0)], tiles=2, heads=2, d=64, axes=(20, 22, 22))
    rows = lambda t: c.view(t, "q").view(4, 6, 2, 64)   # noqa: E731
    rows(c.q[1])[:2, :4].copy_(rows(c.q[0])[2:, 2:])
    c.run()
    assert same(rows(c.q_out[1])[:2, :4].clone(), rows(c.q_out[0])[2:, 2:].clone())


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0), dict(scaling="ramp", factor=2.0, length=64)])
def test_scaled_frequencies(scaling):
    Call(dtype="f32", origin=[(0, 500, 900), (1, 0, 4000)], **scaling).run().check()


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_what_lies_between(dtype, token_major):
    c = Call(pad=24, token_major=token_major, dtype=dtype, heads=5, kv_heads=2, d=80, axes=(16, 16, 16)).run()
    c.check()
    for i in range(2):   # nothing else is written
        for key, ys in (("q", c.q_out), ("k", c.k_out)):
            c.view(ys[i], key).fill_(7.0)
            assert bool((ys[i] == 7.0).all())


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("token_major", [False, True])
def test_in_place(norm, token_major):
    apart = Call(norm=norm, token_major=token_major, heads=7, d=96, axes=(16, 16, 16), layout="half").run()
    c = Call(norm=norm, token_major=token_major, heads=7, d=96, axes=(16, 16, 16), layout="half")
    c.q_out, c.k_out = c.q, c.k
    c.run()
    for a, b in zip(apart.q_out + apart.k_out, c.q + c.k):
        assert same(a, b)


def test_tiles_that_do_not_run_stay():
    flags = torch.arange(70) % 3 != 1
    c = Call(tiles=70, size=(1, 3, 5), heads=2).run(run=flags.to(torch.uint8).cuda())
    c.check([i for i in range(70) if flags[i]])
    for i in range(70):
        if not flags[i]:
            assert bool((c.q_out[i] == 7.0).all()) and bool((c.k_out[i] == 7.0).all())


def test_channels_that_do_not_turn_pass_bit_by_bit():
    for layout, axes in (("half", (16, 0, 0)), ("interleaved", (2, 4, 4))):
        c = Call(d=64, axes=axes, layout=layout, heads=3)
        turned = sum(axes)
        odd = torch.tensor([float("inf"), -float("inf"), 0.0, -0.0, 1e-40, 3e38]).to(torch.bfloat16).cuda()
        for i in range(2):
            c.view(c.q[i], "q")[..., turned:turned + 6] = odd
        c.run()
        for i in range(2):
            assert same(c.view(c.q[i], "q")[..., turned:].clone(), c.view(c.q_out[i], "q")[..., turned:].clone())


@pytest.mark.parametrize("gain", [1e30, 1e-30, 1e19])
def test_norms_of_heads_far_from_one(gain):
    Call(dtype="f32", norm=True, gain=gain, heads=9, d=128, axes=(44, 42, 42), seed=3).run()   # (eps counts below: checked without it)
    c = Call(dtype="f32", norm=True, gain=gain, heads=9, d=128, axes=(44, 42, 42), seed=3)
    c.p.eps = 0.0
    c.run()
    for i in range(2):
        ref, tol = rotary64(c.view(c.q[i], "q").cpu(), c.freq.cpu(), c.coords(i), c.axes, c.layout, c.wq.cpu(), eps=0.0)
        check(c.view(c.q_out[i], "q"), ref, tol, "f32")


def test_nan_stays_in_its_pair_and_with_a_norm_in_its_head():
    for norm in (False, True):
        c = Call(norm=norm, heads=4, d=64, axes=(20, 22, 22))
        c.view(c.q[0], "q")[3, 2, 10] = float("nan")
        c.run()
        bad = torch.isnan(c.view(c.q_out[0], "q")).cpu()
        want = torch.zeros_like(bad)
        want[3, 2, slice(None) if norm else slice(10, 12)] = True
        assert torch.equal(bad, want) and not bool(torch.isnan(c.q_out[1]).any())


def test_only_one_of_two_is_normalised():
    c = Call(norm=True, heads=4, kv_heads=4)
    plain = Call(heads=4, kv_heads=4)
    c.run(k_weight=None)
    plain.q, plain.k = c.q, c.k
    plain.run()
    for i in range(2):
        assert same(c.k_out[i], plain.k_out[i]) and not same(c.q_out[i], plain.q_out[i])


def test_heads_beyond_four_gigabytes():
    n = 5
    c = Call(size=(1, 1, n), heads=2, kv_heads=1, d=64, axes=(0, 0, 64), tiles=1)
    far = (1 << 31) + 4096
    big = torch.empty(far + n * 64, dtype=torch.bfloat16, device="cuda")
    c.p.q_stride_head = c.p.q_out_stride_head = far
    x = torch.randn((2, n, 64)).to(torch.bfloat16)
    for a in range(2):
        big[a * far:a * far + n * 64] = x[a].flatten().cuda()
    c.q, c.q_out = [big], [big]
    c.run()
    ref, tol = rotary64(x.transpose(0, 1), c.freq.cpu(), c.coords(0), c.axes, c.layout)
    check(torch.stack([big[a * far:a * far + n * 64].view(n, 64) for a in range(2)], dim=1), ref, tol, "bf16")


def test_on_another_stream_and_captured():
    eager, graphed = (Call(heads=6, d=128, axes=(44, 42, 42), norm=True, listed=5000, columns=3) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        sg.sg_tile_rotary(graphed.p, graphed.q, graphed.q_out, graphed.freq, k=graphed.k, k_out=graphed.k_out, positions=graphed.positions,
                          q_weight=graphed.wq, k_weight=graphed.wk)
    for step in range(3):
        for c in (eager, graphed):
            for t in c.positions:
                t.add_(17 * step)
            for t in c.q + c.k:
                t.mul_(-0.5)
        eager.run()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.q_out + eager.k_out, graphed.q_out + graphed.k_out):
            assert same(a, b)


def test_scores_depend_on_distances():
    """<turned q, turned k> of two tokens is that of the same two vectors anywhere else at the same distance."""
    g = torch.Generator().manual_seed(9)
    q, k = (torch.randn((1, 64), generator=g).expand(400, 64).contiguous().cuda() for _ in range(2))
    p = sg.make_rotary_problem((1, 20, 20), 1, 64, "f32", (0, 32, 32))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    sg.sg_tile_rotary(p, [q], [qo], sg.sg_rotary_frequencies(p), k=[k], k_out=[ko], origin=[(0, 0, 0)])
    s = (qo.double().cpu() @ ko.double().cpu().t()).view(20, 20, 20, 20)
    # 64 products of numbers of size |q||k|, each off by 2^-20 of it
    tol = 64 * 2.0 ** -20 * float(q.abs().max() * k.abs().max())
    assert float((s[3, 4, 7, 9] - s[13, 14, 17, 19]).abs()) <= tol and float((s[0, 0, 5, 2] - s[14, 17, 19, 19]).abs()) <= tol
    assert float((s[3, 4, 7, 9] - s[7, 9, 3, 4]).abs()) > 1e-3
