"""The operators of a tile's transformer block run one after the other, as a denoising step does: gate, norm, norm of the heads, attention of tile and
text, residual norm, attention to the prompts, residual norm into 8 bits, fuse.  Each operator is held against the 64-bit form of what it was
given, and the whole run, captured, against the eager one."""
import pytest
import torch

import paper_2508_17756_amd as sg
from context_util import TORCH, U8, U16, U32, attend64, bound, norm64
from synthetic.configs import TileGeometry

pytestmark = pytest.mark.gpu

T, TILE, HEADS, D, TEXT, PROMPT = 3, 10, 4, 64, 77, 90
N, C = T * TILE * TILE, HEADS * D
EPS = 1e-6


class Block:
    def __init__(self, dtype, seed=0):
        g = torch.Generator().manual_seed(90 + seed)
        dt = TORCH[dtype]
        self.dtype = dtype
        geom = TileGeometry("block", T, 16, 16, TILE, TILE, 6, 6, 2, 2, HEADS, D, dtype, 1)
        self.tiles = 4
        self.canvas = sg.make_problem(geom)
        new = lambda *shape: torch.zeros(shape, dtype=dt, device="cuda")   # noqa: E731
        rnd = lambda *shape: torch.randn(shape, generator=g).to(dt).to("cuda")   # noqa: E731
        many = lambda make, *shape: [make(*shape) for _ in range(self.tiles)]   # noqa: E731
        self.x, self.cached = many(rnd, N, C), many(rnd, N, C)
        self.w = [1 + 0.1 * rnd(C) for _ in range(3)]
        self.w_head = 1 + 0.1 * rnd(D)
        self.text_k, self.text_v = rnd(TEXT, HEADS, D), rnd(TEXT, HEADS, D)
        prompts = [(rnd(PROMPT, HEADS, D), rnd(PROMPT, HEADS, D)) for _ in range(2)]
        self.prompt_k, self.prompt_v = ([prompts[i % 2][j] for i in range(self.tiles)] for j in range(2))
        self.prompt_len = torch.tensor([PROMPT, 13, 64, 0], dtype=torch.int32, device="cuda")
        self.text_len = torch.tensor([TEXT - 7], dtype=torch.int32, device="cuda")
        self.has = torch.ones(self.tiles, dtype=torch.uint8, device="cuda")
        self.scores = torch.zeros(self.tiles, device="cuda")
        self.run = torch.zeros(self.tiles, dtype=torch.uint8, device="cuda")
        self.y, self.q, self.joint, self.s1, self.y2, self.cross, self.s2 = (many(new, N, C) for _ in range(7))
        self.final = [torch.zeros((N, C), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(self.tiles)]
        self.final_scale = [torch.zeros((N, C // 128), device="cuda") for _ in range(self.tiles)]
        self.packed = many(new, HEADS, N, D)
        self.grid = new(HEADS, T * 16 * 16, D)
        self.norm = sg.make_norm_problem(N, C, dtype, eps=EPS)
        self.norm_head = sg.make_norm_problem(N * HEADS, D, dtype, eps=EPS)
        self.norm_out = sg.make_norm_problem(N, C, dtype, out_dtype="e4m3", scale_group=128, eps=EPS)
        self.p_joint = sg.make_context_problem(N, TEXT, HEADS, D, dtype, own_tokens=N, token_major=True)
        self.p_cross = sg.make_context_problem(N, PROMPT, HEADS, D, dtype, token_major=True)
        n = max(sg.sg_context_workspace_bytes(p, self.tiles) for p in (self.p_joint, self.p_cross))
        self.ws = torch.zeros(n, dtype=torch.uint8, device="cuda")   # the calls follow each other on one stream: one workspace

    def outputs(self):
        return [self.grid, self.run] + [t for name in ("y", "q", "joint", "s1", "y2", "cross", "s2", "final", "final_scale", "packed")
                                        for t in getattr(self, name)]

    def step(self):
        run = self.run
        sg.sg_cache_gate_static(self.x, self.cached, self.has, 0.05, self.scores, run)
        sg.sg_tile_residual_norm(self.norm, self.x, self.w[0], self.y, run=run)
        heads = lambda ts: [t.view(N * HEADS, D) for t in ts]   # noqa: E731
        sg.sg_tile_residual_norm(self.norm_head, heads(self.y), self.w_head, heads(self.q), run=run)
        # (keys and values are the norms themselves: what a projection does is no part of this)
        sg.sg_tile_prefix_attention(self.p_joint, self.q, self.q, self.y, self.text_k, self.text_v, self.joint, prefix_len=self.text_len,
                                    run=run, workspace=self.ws)
        sg.sg_tile_residual_norm(self.norm, self.joint, self.w[1], self.y2, residual=self.x, sum_out=self.s1, run=run)
        sg.sg_tile_cross_attention(self.p_cross, self.y2, self.prompt_k, self.prompt_v, self.cross, ctx_len=self.prompt_len, run=run,
                                   workspace=self.ws)
        sg.sg_tile_residual_norm(self.norm_out, self.cross, self.w[2], self.final, residual=self.s1, sum_out=self.s2, out_scale=self.final_scale,
                                 run=run)
        for s, t in zip(self.s2, self.packed):   # the tiles that were skipped still hold the last step's
            t.copy_(s.view(N, HEADS, D).transpose(0, 1))
        sg.sg_tile_blend(self.canvas, self.packed, self.grid)

    def check(self, i):
        u = U16 if self.dtype == "bf16" else U32
        cpu = lambda t: t.cpu().double()   # noqa: E731
        scale = float(torch.tensor(D ** -0.5, dtype=torch.float32))

        def norm(x, r, w, got, s=None):
            total, y = norm64(x, r, w, EPS)
            mag = x.abs() + (0 if r is None else r.abs())
            if s is not None:
                assert bool(((s - total).abs() <= u * total.abs() + U32 * mag + 1e-30).all())
            rel = (x.shape[1] / 4 + 16) * U32
            tol = rel * y.abs() + 2 * U32 * (y / total.where(total != 0, torch.ones_like(total))).abs() * mag
            if got is not None:
                assert bool(((got - y).abs() <= tol + u * y.abs() * (1 + 2 * rel) + 1e-30).all())
            return y, tol

        norm(cpu(self.x[i]), None, cpu(self.w[0]), cpu(self.y[i]))
        norm(cpu(self.y[i]).view(-1, D), None, cpu(self.w_head), cpu(self.q[i]).view(-1, D))
        n_text, n_prompt = int(self.text_len[0]), int(self.prompt_len[i])
        for a in range(HEADS):
            of = lambda t: cpu(t).view(-1, HEADS, D)[:, a]   # noqa: E731
            k = torch.cat([of(self.text_k)[:n_text], of(self.q[i])])
            v = torch.cat([of(self.text_v)[:n_text], of(self.y[i])])
            o, mag, s = attend64(of(self.q[i]), k, v, scale)
            assert bool(((of(self.joint[i]) - o).abs() <= bound(o, mag, s, D, k.shape[0], self.dtype)).all())
            o, mag, s = attend64(of(self.y2[i]), of(self.prompt_k[i])[:n_prompt], of(self.prompt_v[i])[:n_prompt], scale)
            assert bool(((of(self.cross[i]) - o).abs() <= bound(o, mag, s, D, n_prompt, self.dtype)).all())
        norm(cpu(self.joint[i]), cpu(self.x[i]), cpu(self.w[1]), cpu(self.y2[i]), cpu(self.s1[i]))
        y, tol = norm(cpu(self.cross[i]), cpu(self.s1[i]), cpu(self.w[2]), None, cpu(self.s2[i]))
        sc = cpu(self.final_scale[i])[..., None]
        blocks = y.view(N, -1, 128)
        deq = self.final[i].cpu().float().double().view(N, -1, 128) * sc
        assert bool(((deq - blocks).abs() <= tol.view(blocks.shape) * (1 + U8) + (U8 + 8 * U32) * blocks.abs() + 2.0 ** -10 * sc + 1e-30).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_block_of_operators(dtype):
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
def test_a_captured_block(dtype):
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
            b.prompt_len.fill_(20 * k)
        eager.step()
        g.replay()
        torch.cuda.synchronize()
        assert eager.run.tolist() == [int((i + k) % 3 != 0) for i in range(4)]
        for x, y in zip(eager.outputs(), graphed.outputs()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
