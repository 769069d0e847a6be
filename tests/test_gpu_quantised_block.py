"""The quantised half of a tile's transformer block, run as a denoising step does: gate, norm into 8-bit integers, projection to queries, keys and values, rotary
positions with the norm of the heads, attention of tile and text, the output projection, gated residual norm into 8-bit integers, the feed-forward block with
GELU, gate and residual, fuse.  Each operator is held against the 64-bit form of what it was given, and the whole run, captured, against the eager one."""
import pytest
import torch

import paper_2508_17756_amd as sg
from block_util import TORCH, check, check_eight, gated64, linear64, rotary64
from context_util import attend64, bound
from synthetic.configs import TileGeometry

pytestmark = pytest.mark.gpu

T, TILE, CANVAS, HEADS, D, TEXT, WIDE = 3, 10, 16, 4, 64, 45, 528
N, C = T * TILE * TILE, HEADS * D
AXES = (16, 24, 24)
EPS = 1e-6


class Block:
    def __init__(self, dtype, seed=0):
        g = torch.Generator().manual_seed(170 + seed)
        dt = TORCH[dtype]
        self.dtype, self.tiles = dtype, 4
        geom = TileGeometry("block", T, CANVAS, CANVAS, TILE, TILE, 6, 6, 2, 2, HEADS, D, dtype, 1)
        self.canvas = sg.make_problem(geom)
        new = lambda *shape, kind=dt: [torch.zeros(shape, dtype=kind, device="cuda") for _ in range(self.tiles)]   # noqa: E731
        rnd = lambda *shape, size=1.0, kind=dt: (size * torch.randn(shape, generator=g)).to(kind).cuda()   # noqa: E731

        def weights(outputs, channels):
            w = torch.randn((outputs, channels), generator=g)
            scale = w.abs().amax(dim=1) / 127
            return torch.round(w / scale[:, None]).to(torch.int8).cuda(), (scale / channels ** 0.5).cuda(), rnd(outputs, size=0.1)

        self.x, self.cached = [rnd(N, C) for _ in range(self.tiles)], [rnd(N, C) for _ in range(self.tiles)]
        self.mods = [[rnd(1, C, size=0.3, kind=torch.float32) for _ in range(self.tiles)] for _ in range(6)]   # shift, scale, gate: twice, a vector per tile
        self.qkv_w, self.out_w, self.up_w, self.down_w = weights(3 * C, C), weights(C, C), weights(WIDE, C), weights(C, WIDE)
        self.wq, self.wk = 1 + rnd(D, size=0.1), 1 + rnd(D, size=0.1)
        self.text_k, self.text_v = rnd(TEXT, HEADS, D), rnd(TEXT, HEADS, D)
        self.has, self.run = torch.ones(4, dtype=torch.uint8, device="cuda"), torch.zeros(4, dtype=torch.uint8, device="cuda")
        self.scores = torch.zeros(4, device="cuda")
        self.n1, self.n2, self.n3 = new(N, C, kind=torch.int8), new(N, C, kind=torch.int8), new(N, C, kind=torch.int8)
        self.h8 = new(N, WIDE, kind=torch.int8)
        self.s1, self.s2, self.s3, self.sh = (new(N, 1, kind=torch.float32) for _ in range(4))
        self.qkv, self.q, self.k, self.joint, self.proj, self.mid, self.h, self.down, self.y, self.unused = \
            new(N, 3 * C), new(N, C), new(N, C), new(N, C), new(N, C), new(N, C), new(N, WIDE), new(N, C), new(N, C), new(N, C)
        self.packed = new(HEADS, N, D)
        self.grid = torch.zeros((HEADS, T * CANVAS * CANVAS, D), dtype=dt, device="cuda")
        self.norm = sg.make_gated_norm_problem(N, C, dtype, out_dtype="int8", norm="layer", mod_dtype="f32", eps=EPS)
        self.quantise = sg.make_gated_norm_problem(N, C, dtype, out_dtype="int8", norm="rms", eps=EPS)
        self.quantise_wide = sg.make_gated_norm_problem(N, WIDE, dtype, out_dtype="int8", norm="rms", eps=EPS)
        self.last = sg.make_gated_norm_problem(N, C, dtype, norm="rms", mod_dtype="f32", eps=EPS)
        lin = lambda k, m, act=None: sg.make_int8_linear_problem(N, k, m, dtype, activation=act)   # noqa: E731
        self.p_qkv, self.p_out, self.p_up, self.p_down = lin(C, 3 * C), lin(C, C), lin(C, WIDE, "gelu"), lin(WIDE, C)
        self.rot = sg.make_rotary_problem((T, TILE, TILE), HEADS, D, dtype, AXES, wrap=(T, CANVAS, CANVAS), eps=EPS, token_major=True)
        self.rot.q_stride_token = self.rot.k_stride_token = 3 * C   # queries and keys lie side by side as the projection leaves them
        self.freq = sg.sg_rotary_frequencies(self.rot)
        self.origin = [(0, 6 * (i // 2) + 9, 6 * (i % 2) + 9) for i in range(4)]   # a shifted partition: the last tiles wrap around
        self.joint_p = sg.make_context_problem(N, TEXT, HEADS, D, dtype, own_tokens=N, token_major=True)
        self.joint_p.own_stride_token = C
        self.v = new(N, C)
        self.ws = torch.zeros(max(1, sg.sg_context_workspace_bytes(self.joint_p, 4)), dtype=torch.uint8, device="cuda")

    def outputs(self):
        return [self.grid, self.run] + [t for name in ("n1", "s1", "qkv", "q", "k", "joint", "n2", "s2", "proj", "mid", "n3", "s3", "h", "h8", "sh", "down", "y", "unused",
                                                       "packed") for t in getattr(self, name)]

    def step(self):
        run = self.run
        sg.sg_cache_gate_static(self.x, self.cached, self.has, 0.05, self.scores, run)
        shift, scale, gate, shift2, scale2, gate2 = self.mods
        sg.sg_tile_gated_norm(self.norm, self.x, self.n1, scale=scale, shift=shift, out_scale=self.s1, run=run)
        sg.sg_tile_int8_linear(self.p_qkv, self.n1, self.s1, self.qkv_w[0], self.qkv_w[1], self.qkv, bias=self.qkv_w[2], run=run)
        part = lambda j: [t[:, j * C:] for t in self.qkv]   # noqa: E731
        sg.sg_tile_rotary(self.rot, part(0), self.q, self.freq, k=part(1), k_out=self.k, origin=self.origin, q_weight=self.wq, k_weight=self.wk, run=run)
        for v, t in zip(self.v, self.qkv):
            v.copy_(t[:, 2 * C:])
        sg.sg_tile_prefix_attention(self.joint_p, self.q, self.k, self.v, self.text_k, self.text_v, self.joint, run=run, workspace=self.ws)
        sg.sg_tile_gated_norm(self.quantise, self.joint, self.n2, out_scale=self.s2, run=run)
        sg.sg_tile_int8_linear(self.p_out, self.n2, self.s2, self.out_w[0], self.out_w[1], self.proj, bias=self.out_w[2], run=run)
        sg.sg_tile_gated_norm(self.norm, self.proj, self.n3, residual=self.x, gate=gate, scale=scale2, shift=shift2, sum_out=self.mid, out_scale=self.s3, run=run)
        sg.sg_tile_int8_linear(self.p_up, self.n3, self.s3, self.up_w[0], self.up_w[1], self.h, bias=self.up_w[2], run=run)
        sg.sg_tile_gated_norm(self.quantise_wide, self.h, self.h8, out_scale=self.sh, run=run)
        sg.sg_tile_int8_linear(self.p_down, self.h8, self.sh, self.down_w[0], self.down_w[1], self.down, run=run)
        sg.sg_tile_gated_norm(self.last, self.down, self.unused, residual=self.mid, gate=gate2, sum_out=self.y, run=run)
        for s, t in zip(self.y, self.packed):
            t.copy_(s.view(N, HEADS, D).transpose(0, 1))
        sg.sg_tile_blend(self.canvas, self.packed, self.grid)

    def check(self, i):
        cpu = lambda ts: ts[i].cpu()   # noqa: E731
        shift, scale, gate, shift2, scale2, gate2 = (m[i].cpu() for m in self.mods)
        w = lambda ws: [t.cpu() for t in ws]   # noqa: E731

        def norm(x, r, gate, scale, shift, kind, out=None, out_scale=None, total=None):
            s, es, y, ey = gated64(cpu(x), None if r is None else cpu(r), gate, None, None, scale, shift, kind, "none", 1.0, 0, EPS)
            if total is not None:
                check(cpu(total), s, es, self.dtype)
            if out_scale is not None:
                check_eight(cpu(out), cpu(out_scale), y, ey, "int8", 0)
            elif out is not None:
                check(cpu(out), y, ey, self.dtype)

        def linear(x, s, ws, out, bias=True, gelu=False):
            wi, wsc, b = w(ws)
            ref, tol = linear64(cpu(x), cpu(s).flatten(), wi, wsc, b if bias else None, gelu)
            check(cpu(out), ref, tol, self.dtype)

        norm(self.x, None, None, scale, shift, "layer", self.n1, self.s1)
        linear(self.n1, self.s1, self.qkv_w, self.qkv)
        at = torch.arange(N)
        coords = torch.stack([at // (TILE * TILE), (self.origin[i][1] + at // TILE % TILE) % CANVAS, (self.origin[i][2] + at % TILE) % CANVAS], dim=1)
        for j, (out, weight) in enumerate(((self.q, self.wq), (self.k, self.wk))):
            ref, tol = rotary64(cpu(self.qkv)[:, j * C:(j + 1) * C].reshape(N, HEADS, D), self.freq.cpu(), coords, AXES, "interleaved", weight.cpu(), EPS)
            check(cpu(out).view(N, HEADS, D), ref, tol, self.dtype)
        soft = float(torch.tensor(D ** -0.5, dtype=torch.float32))
        for a in range(HEADS):
            of = lambda t: t.cpu().double().view(-1, HEADS, D)[:, a]   # noqa: E731
            o, mag, s = attend64(of(self.q[i]), torch.cat([of(self.text_k), of(self.k[i])]), torch.cat([of(self.text_v), of(self.v[i])]), soft)
            assert bool(((of(self.joint[i]) - o).abs() <= bound(o, mag, s, D, TEXT + N, self.dtype)).all())
        norm(self.joint, None, None, None, None, "rms", self.n2, self.s2)
        linear(self.n2, self.s2, self.out_w, self.proj)
        norm(self.proj, self.x, gate, scale2, shift2, "layer", self.n3, self.s3, self.mid)
        linear(self.n3, self.s3, self.up_w, self.h, gelu=True)
        norm(self.h, None, None, None, None, "rms", self.h8, self.sh)
        linear(self.h8, self.sh, self.down_w, self.down, bias=False)
        norm(self.down, self.mid, gate2, None, None, "rms", self.unused, None, self.y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_quantised_block(dtype):
    b = Block(dtype)
    b.step()
    torch.cuda.synchronize()
    assert b.run.tolist() == [1] * 4
    for i in range(4):
        b.check(i)
    # the next step: two tiles have hardly moved and keep what they have
    before = [t.clone() for t in b.outputs()]
    for i in range(4):
        b.cached[i].copy_(b.x[i])
    for i in (1, 2):
        b.x[i].mul_(0.5)
    b.step()
    torch.cuda.synchronize()
    assert b.run.tolist() == [0, 1, 1, 0]
    for i in (1, 2):
        b.check(i)
    for k, (now, was) in enumerate(zip(b.outputs(), before)):
        if k >= 2 and (k - 2) % 4 in (0, 3):
            assert torch.equal(now.view(torch.uint8), was.view(torch.uint8)), k
    assert not torch.equal(b.grid, before[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_quantised_block(dtype):
    eager, graphed = Block(dtype, seed=1), Block(dtype, seed=1)
    eager.step()
    graphed.step()
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        graphed.step()
    torch.cuda.synchronize()
    for k in range(4):
        for b in (eager, graphed):
            for i in range(4):
                b.cached[i].copy_(b.x[i])
                if (i + k) % 3 != 0:
                    b.x[i].mul_(0.75)
        eager.step()
        g.replay()
        torch.cuda.synchronize()
        assert eager.run.tolist() == [int((i + k) % 3 != 0) for i in range(4)]
        for x, y in zip(eager.outputs(), graphed.outputs()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
