"""Plain 64-bit forms of context attention and the residual norm, and how far a kernel may be from them (not a test module).

Half a step of the types (torch.finfo(t).eps / 2, relative): fp32 2^-24, bf16 2^-8, e4m3 2^-4.
"""
import math

import torch

import paper_2508_17756_amd as sg

U32, U16, U8 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def attend64(q, k, v, scale):
    """One head, [n, d] and [m, d] in fp64: (o, a, s): the result, the same of |v|, and max over keys of scale * sum |q||k|."""
    if k.shape[0] == 0:
        z = torch.zeros_like(q)
        return z, z, torch.zeros(q.shape[0], 1, dtype=torch.float64, device=q.device)
    w = torch.softmax((q * scale) @ k.t().contiguous(), dim=-1)
    return w @ v, w @ v.abs(), (scale * (q.abs() @ k.abs().t().contiguous())).amax(dim=1, keepdim=True)


def bound(o, a, s, d, keys, dtype):
    """Elementwise error of the kernels.  A score is off by at most (d + 2) 2^-24 of scale sum|q||k| (products and their sum), its exponent's
    argument by 4 roundings of at most twice that size more; a probability by as much, relatively, and by 2^-21 of the exponential.  Their
    sums over the keys, and the references' changes, at most (keys + 64) 2^-24.  Numerator and denominator both: times two.  bf16
    rounds each probability and the result once more."""
    rel = 2 * ((d + 2 + 8) * U32 * s + (keys + 64) * U32 + 2.0 ** -21)
    return (rel + (U16 if dtype == "bf16" else 0.0)) * a + (U16 if dtype == "bf16" else U32) * o.abs() + 1e-30


class Call:
    """Tensors of one context attention and its 64-bit result.  lay: "packed", "token" (token-major) or "odd" (padded strides)."""

    def __init__(self, tiles, tokens, heads, kv_heads, d, dtype, ctx, own=0, prefix=False, lay="packed", ragged=False, masked=False,
                 run=False, seed=0, spread=1.0, device="cuda"):
        self.tiles, self.tokens, self.heads, self.kv_heads, self.d, self.dtype = tiles, tokens, heads, kv_heads, d, dtype
        self.ctx, self.own, self.prefix, self.lay, self.device = ctx, own, prefix, lay, device
        g = torch.Generator().manual_seed(1234 + seed)
        self.gen = g
        self.q = [self._tensor(heads, tokens, spread) for _ in range(tiles)]
        keys = own if prefix else ctx
        self.k = [self._tensor(kv_heads, keys, spread) for _ in range(tiles)]
        self.v = [self._tensor(kv_heads, keys) for _ in range(tiles)]
        if prefix:
            self.pk, self.pv = self._tensor(kv_heads, ctx, spread), self._tensor(kv_heads, ctx)
        self.out = [self._tensor(heads, tokens) for _ in range(tiles)]
        self.lens = None
        if ragged:   # the first whole, the second empty
            self.lens = torch.randint(0, keys + 1, (tiles,), generator=g, dtype=torch.int32)
            self.lens[0] = keys
            if tiles > 1:
                self.lens[1] = 0
        self.mask = (torch.rand((tiles, ctx), generator=g) < 0.7).to(torch.uint8) if masked else None
        if masked:
            self.mask[-1] = 0 if tiles > 1 else self.mask[-1]
        self.run = None
        if run:
            self.run = (torch.arange(tiles) % 3 != 1).to(torch.uint8)
        self.p = sg.make_context_problem(tokens, ctx, heads, d, dtype, kv_heads=kv_heads, own_tokens=own, token_major=lay == "token")
        if lay == "odd":
            for name, n in (("q", tokens), ("ctx", ctx), ("own", own), ("out", tokens)):
                setattr(self.p, name + "_stride_token", d + 24)
                setattr(self.p, name + "_stride_head", (n + 3) * (d + 24) + 8)

    def _tensor(self, heads, n, spread=1.0):
        """[heads, n, d] view of N(0, spread) values in the layout; what the strides skip holds NaN."""
        d = self.d
        x = (torch.randn((heads, n, d), generator=self.gen) * spread).to(TORCH[self.dtype])
        if self.lay == "packed":
            return x.to(self.device)
        if self.lay == "token":
            return x.transpose(0, 1).contiguous().to(self.device).transpose(0, 1)
        head = (n + 3) * (d + 24) + 8
        flat = torch.full((heads * head,), float("nan"), dtype=x.dtype)
        view = flat.as_strided((heads, n, d), (head, d + 24, 1))
        view.copy_(x)
        return flat.to(self.device).as_strided((heads, n, d), (head, d + 24, 1))

    def workspace(self):
        return torch.empty(sg.sg_context_workspace_bytes(self.p, self.tiles), dtype=torch.uint8, device=self.device)

    def __call__(self, workspace=None, out=None):
        dev = lambda t: None if t is None else t.to(self.device)   # noqa: E731
        ws = self.workspace() if workspace is None else workspace
        out = self.out if out is None else out
        if self.prefix:
            sg.sg_tile_prefix_attention(self.p, self.q, self.k if self.own else None, self.v if self.own else None, self.pk, self.pv, out,
                                        own_len=dev(self.lens), prefix_len=dev(getattr(self, "prefix_len", None)), run=dev(self.run),
                                        workspace=ws)
        else:
            sg.sg_tile_cross_attention(self.p, self.q, self.k, self.v, out, ctx_len=dev(self.lens), key_mask=dev(self.mask),
                                       run=dev(self.run), workspace=ws)
        return out

    def keys(self, i):
        """Indices of the keys of tile i that count."""
        n = self.own if self.prefix else self.ctx
        keep = torch.ones(n, dtype=torch.bool)
        if self.lens is not None:
            keep &= torch.arange(n) < int(self.lens[i])
        if self.mask is not None:
            keep &= self.mask[i] != 0
        return torch.nonzero(keep)[:, 0]

    def reference(self, i, a):
        """(o, bound) of head a of tile i."""
        b = a // (self.heads // self.kv_heads)
        at = self.keys(i)
        k, v = self.k[i][b].cpu().double()[at], self.v[i][b].cpu().double()[at]
        if self.prefix:
            n = self.ctx if getattr(self, "prefix_len", None) is None else max(0, min(self.ctx, int(self.prefix_len)))
            k = torch.cat([self.pk[b].cpu().double()[:n], k])
            v = torch.cat([self.pv[b].cpu().double()[:n], v])
        scale = float(torch.tensor(self.p.scale, dtype=torch.float32))
        o, mag, s = attend64(self.q[i][a].cpu().double(), k, v, scale)
        return o, bound(o, mag, s, self.d, k.shape[0], self.dtype)

    def check(self, out=None, before=None, heads=None):
        out = self.out if out is None else out
        for i in range(self.tiles):
            if self.run is not None and int(self.run[i]) == 0:
                assert torch.equal(out[i].cpu(), before[i].cpu()), "tile %d does not run and was written" % i
                continue
            for a in range(self.heads) if heads is None else heads:
                o, tol = self.reference(i, a)
                err = (out[i][a].cpu().double() - o).abs()
                assert bool((err <= tol).all()), "tile %d head %d: %.3e of the bound" % (i, a, float((err / tol).max()))


def norm64(x, residual, weight, eps):
    s = x.double() if residual is None else x.double() + residual.double()
    y = s / torch.sqrt(s.square().mean(dim=-1, keepdim=True) + eps)
    return s, y if weight is None else y * weight.double()


def log2_range(v):
    return math.log2(float(v.abs().max()))
