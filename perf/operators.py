"""The operators of a tile's transformer block beside its self-attention, as cases that can be timed and compared.

A case is a dict of plain values.  Kinds:
  cross    sg_tile_cross_attention    queries of every tile over an encoder's states (its own context, with a length, padded places masked)
  prefix   sg_tile_prefix_attention   queries of every tile over a prefix that all tiles share, and then over the tile's own keys
  norm     sg_tile_residual_norm      s = x + residual, root-mean-square norm of s with a weight, in the tensors' type or in e4m3 with scales

`run` computes them with elementary torch operations in fp32, or, where `own` is set, calls the library.  Sizes are those of the benchmark
configurations (21 x 45 x 80 = 75,600 tokens, 40 heads x 128; previews of fewer frames; 48 heads x 64) and generic odd ones; values are
N(0, 1), like the projections of a normalised hidden state.
"""
import math

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0


def _cross(name, tiles, tokens, heads, d, ctx, dtype="bf16", kv_heads=None, **options):
    c = {"kind": "cross", "tiles": tiles, "tokens": tokens, "heads": heads, "kv_heads": kv_heads or heads, "d": d, "ctx": ctx, "dtype": dtype}
    if name:
        c["name"] = name
    c.update(options)
    return c


def _prefix(name, tiles, tokens, own_tokens, heads, d, prefix, dtype="bf16", kv_heads=None, **options):
    c = {"kind": "prefix", "tiles": tiles, "tokens": tokens, "own": own_tokens, "heads": heads, "kv_heads": kv_heads or heads, "d": d,
         "prefix": prefix, "dtype": dtype}
    if name:
        c["name"] = name
    c.update(options)
    return c


def _norm(name, tiles, rows, channels, dtype="bf16", out="same", group=0, residual=True):
    c = {"kind": "norm", "tiles": tiles, "rows": rows, "channels": channels, "dtype": dtype, "out": out, "group": group, "residual": residual}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token over a short prompt: nothing but latency
        _cross("cross_token", 1, 1, 8, 64, 77),
        # fp32 at a preview size: a caller checking a bf16 run against full precision
        _cross("cross_f32_preview", 4, 2880, 8, 128, 226, "f32"),
        # one frame of the 2K tiling: nine tiles, each with a prompt of its own, padded to 512; queries as the projection leaves them
        _cross("cross_regional_2k", 9, 3840, 40, 128, 512, token_major=True, ragged=True, masked=True),
        # 48 heads x 64 over a prompt of 226 tokens, four non-overlapping tiles
        _cross("cross_heads64", 4, 17550, 48, 64, 226),
        # the headline tile over a prompt of 512 tokens
        _cross("cross_tile720p", 1, 75600, 40, 128, 512),
        # the smallest joint call: four fp32 tiles of 300 tokens over a shared prompt
        _prefix("prefix_f32_tiny", 4, 300, 300, 2, 64, 77, "f32"),
        # twenty requests of one token each, grouped heads, over 32,760 tokens that they share and some of their own
        _prefix("prefix_single_tokens", 20, 1, 460, 40, 128, 32760, kv_heads=8, ragged=True),
        # joint attention, 48 heads x 64: text and tile in one softmax
        _prefix("prefix_joint64", 4, 2925, 2925, 48, 64, 226),
        # joint attention of nine ordinary tiles with a long shared prompt; the largest amount of arithmetic
        _prefix("prefix_joint_9tiles", 9, 3840, 3840, 24, 128, 512),
        # one row, in fp32, quantised by blocks of 128 channels for the next projection
        _norm("norm_row_f32", 1, 1, 5120, "f32", "e4m3", 128),
        # norm of queries (or keys) per head before attention: short rows
        _norm("norm_heads_9tiles", 9, 3840 * 40, 128, residual=False),
        # residual stream of the headline tile, quantised by rows for the next projection
        _norm("norm_tile720p", 1, 75600, 5120, "bf16", "e4m3", 0),
    ]


def _spread(rng, low, high):
    """An integer whose logarithm is spread evenly over [low, high]."""
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["cross", "cross", "prefix", "prefix", "prefix", "norm"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "norm":
        rows_of_heads = rng.random() < 0.3
        channels = rng.choice([64, 128]) if rows_of_heads else 8 * _spread(rng, 16, 1024)
        tiles = rng.choice([1, 1, 2, 4, 9, 20])
        rows = _spread(rng, 1, max(1, int(1.5e8 / channels / tiles)))
        out = rng.choice(["same", "e4m3"])
        group = 128 if out == "e4m3" and channels % 128 == 0 and rng.random() < 0.5 else 0
        return _norm(None, tiles, rows, channels, dtype, out, group, not rows_of_heads)
    d = rng.choice([64, 128, 128])
    heads = rng.choice([1, 2, 5, 8, 12, 16, 40])
    kv_heads = rng.choice([n for n in range(1, heads + 1) if heads % n == 0]) if rng.random() < 0.4 else heads
    tiles = rng.choice([1, 2, 4, 9, 20])
    flops, scores = (4e10, 2e9) if dtype == "f32" else (7e11, 1.2e10)   # bounds on the arithmetic and on the bytes of all scores in fp32
    serving = kind == "prefix" and rng.random() < 0.5 or kind == "cross" and rng.random() < 0.2
    if kind == "cross":
        ctx = _spread(rng, 1, 4000)
        top = min(flops / (4.0 * tiles * heads * d * ctx), scores / (4.0 * tiles * heads * ctx), 75600.0)
        tokens = _spread(rng, 1, 16) if serving else _spread(rng, 16, max(17, int(top)))
        return _cross(None, tiles, tokens, heads, d, ctx, dtype, kv_heads, token_major=rng.random() < 0.4,
                      ragged=rng.random() < 0.5, masked=rng.random() < 0.3)
    if serving:
        prefix, tokens, own_tokens = _spread(rng, 64, 60000), _spread(rng, 1, 16), _spread(rng, 1, 2000)
    else:
        prefix = _spread(rng, 1, 2000)
        top = min(flops / (4.0 * tiles * heads * d), scores / (4.0 * tiles * heads))   # bounds tokens * (prefix + tokens)
        tokens = _spread(rng, 16, max(17, int((math.sqrt(prefix * prefix + 4.0 * top) - prefix) / 2)))
        own_tokens = tokens
    return _prefix(None, tiles, tokens, own_tokens, heads, d, prefix, dtype, kv_heads, token_major=rng.random() < 0.3,
                   ragged=serving and rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ states
def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _queries_shape(c):
    n, a, d = c["tokens"], c["heads"], c["d"]
    return (c["tiles"], n, a, d) if c.get("token_major") else (c["tiles"], a, n, d)


def _keys_shape(c, tiles, tokens):
    return (tiles, tokens, c["kv_heads"], c["d"]) if c.get("token_major") else (tiles, c["kv_heads"], tokens, c["d"])


def _lengths(n, most, gen):
    """n lengths of at most `most`, the first of them whole."""
    got = torch.randint(max(1, most // 4), most + 1, (n,), device=DEV, generator=gen, dtype=torch.int32)
    got[0] = most
    return got


def prepare(case, seed):
    c, dt = case, _type(case)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1000 + 17)

    def randn(*shape):
        return torch.randn(shape, dtype=dt, device=DEV, generator=gen)

    s = {"case": c}
    if c["kind"] == "norm":
        t, n, m = c["tiles"], c["rows"], c["channels"]
        s["x"] = randn(t, n, m)
        s["residual"] = randn(t, n, m) if c["residual"] else None
        s["weight"] = 1 + 0.1 * randn(m)
        s["sum"] = torch.empty_like(s["x"]) if c["residual"] else None
        s["out"] = torch.empty((t, n, m), dtype=torch.float8_e4m3fn if c["out"] == "e4m3" else dt, device=DEV)
        s["scale"] = torch.empty((t, n, m // c["group"] if c["group"] else 1), dtype=torch.float32, device=DEV) if c["out"] == "e4m3" else None
    else:
        t = c["tiles"]
        s["q"] = randn(*_queries_shape(c))
        s["out"] = torch.empty_like(s["q"])
        keys = c["ctx"] if c["kind"] == "cross" else c["own"]
        s["k"], s["v"] = randn(*_keys_shape(c, t, keys)), randn(*_keys_shape(c, t, keys))
        s["len"] = _lengths(t, keys, gen) if c.get("ragged") else None
        if c["kind"] == "cross":
            s["mask"] = (torch.rand((t, keys), device=DEV, generator=gen) < 0.9).to(torch.uint8) if c.get("masked") else None
        else:
            s["pk"], s["pv"] = randn(*_keys_shape(c, 1, c["prefix"]))[0], randn(*_keys_shape(c, 1, c["prefix"]))[0]
    if own:   # what a program keeps from call to call: the problem, the tiles' buffers, the workspace
        import paper_2508_17756_amd as sg
        s["sg"] = sg
        s["tiles"] = {key: [None if v is None else v[i] for i in range(c["tiles"])] for key, v in s.items()
                      if key in ("x", "residual", "sum", "out", "scale", "q", "k", "v") and v is not None}
        if c["kind"] == "norm":
            s["p"] = sg.make_norm_problem(c["rows"], c["channels"], c["dtype"], out_dtype="e4m3" if c["out"] == "e4m3" else None,
                                          scale_group=c["group"])
        else:
            ctx, own_tokens = (c["ctx"], 0) if c["kind"] == "cross" else (c["prefix"], c["own"])
            s["p"] = sg.make_context_problem(c["tokens"], ctx, c["heads"], c["d"], c["dtype"], kv_heads=c["kv_heads"], own_tokens=own_tokens,
                                             token_major=bool(c.get("token_major")))
            s["ws"] = torch.empty(sg.sg_context_workspace_bytes(s["p"], c["tiles"]), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _grouped(x, c):
    """Queries as [tiles][kv_heads][heads of the group * tokens][d] in fp32."""
    if c.get("token_major"):
        x = x.transpose(1, 2)
    return x.float().reshape(c["tiles"], c["kv_heads"], -1, c["d"])


def _headed(x, c):
    """Keys or values as [...][kv_heads][tokens][d] in fp32."""
    return (x.transpose(-3, -2) if c.get("token_major") else x).float().contiguous()


def _valid(n, lengths, mask):
    """Which of n keys count, per tile: [tiles][1][1][n], or None where all do."""
    keep = None
    if lengths is not None:
        keep = torch.arange(n, device=DEV)[None, :] < lengths[:, None]
    if mask is not None:
        keep = mask != 0 if keep is None else keep & (mask != 0)
    return None if keep is None else keep[:, None, None, :]


def _ungrouped(o, c):
    o = o.reshape(c["tiles"], c["heads"], c["tokens"], c["d"])
    return (o.transpose(1, 2) if c.get("token_major") else o).to(_type(c)).contiguous()


def _plain_attention(s, c):
    scale = 1.0 / math.sqrt(c["d"])
    q, k, v = _grouped(s["q"], c), _headed(s["k"], c), _headed(s["v"], c)
    keep = _valid(k.shape[2], s["len"], s.get("mask"))
    w = torch.matmul(q, k.transpose(-1, -2)) * scale
    if keep is not None:
        w = torch.where(keep, w, -math.inf)
        v = torch.where(keep.transpose(-1, -2), v, 0.0)
    if c["kind"] == "prefix":
        pk, pv = _headed(s["pk"], c), _headed(s["pv"], c)
        w = torch.cat([torch.matmul(q, pk.transpose(-1, -2)) * scale, w], dim=-1)
    w = torch.exp(w - torch.clamp(w.amax(dim=-1, keepdim=True), min=-3e38))
    total = w.sum(dim=-1, keepdim=True)
    if c["kind"] == "prefix":
        n = c["prefix"]
        o = torch.matmul(w[..., :n], pv) + torch.matmul(w[..., n:], v)
    else:
        o = torch.matmul(w, v)
    return _ungrouped(torch.where(total > 0, o / total, 0.0), c)


def _plain_norm(s, c):
    x = s["x"].float()
    if c["residual"]:
        x = x + s["residual"].float()
    y = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + 1e-6) * s["weight"].float()
    if c["out"] == "same":
        return {"out": y.to(_type(c)), **({"sum": x.to(_type(c))} if c["residual"] else {})}
    blocks = y.reshape(y.shape[0], y.shape[1], -1, c["group"] or c["channels"])
    scale = blocks.abs().amax(dim=-1, keepdim=True) / E4M3_MAX
    q = torch.where(scale > 0, blocks / scale, 0.0).to(torch.float8_e4m3fn).reshape(y.shape)
    return {"out": q, "scale": scale.squeeze(-1), **({"sum": x.to(_type(c))} if c["residual"] else {})}


def run(s):
    c = s["case"]
    if not own:
        return _plain_norm(s, c) if c["kind"] == "norm" else _plain_attention(s, c)
    sg, t = s["sg"], s["tiles"]
    if c["kind"] == "norm":
        sg.sg_tile_residual_norm(s["p"], t["x"], s["weight"], t["out"], residual=t.get("residual"), sum_out=t.get("sum"), out_scale=t.get("scale"))
        return {k: s[k] for k in ("out", "scale", "sum") if s[k] is not None}
    if c["kind"] == "cross":
        sg.sg_tile_cross_attention(s["p"], t["q"], t["k"], t["v"], t["out"], ctx_len=s["len"], key_mask=s["mask"], workspace=s["ws"])
    else:
        sg.sg_tile_prefix_attention(s["p"], t["q"], t["k"], t["v"], s["pk"], s["pv"], t["out"], own_len=s["len"], workspace=s["ws"])
    return s["out"]


# ------------------------------------------------------------------------------------------------ work
def work(case):
    """Each input read once, each output written once; the two products of attention, over all keys that the buffers hold."""
    c, e = case, 4 if case["dtype"] == "f32" else 2
    if c["kind"] == "norm":
        n = c["tiles"] * c["rows"] * c["channels"]
        per = e * (3 if c["residual"] else 1) + (1 if c["out"] == "e4m3" else e)
        scales = 4 * c["tiles"] * c["rows"] * (c["channels"] // c["group"] if c["group"] else 1) if c["out"] == "e4m3" else 0
        return {"bytes": n * per + c["channels"] * e + scales, "flops": 0}
    rows, kv = c["tiles"] * c["tokens"] * c["heads"] * c["d"], c["kv_heads"] * c["d"]
    if c["kind"] == "cross":
        return {"bytes": e * (2 * rows + 2 * c["tiles"] * c["ctx"] * kv) + c["tiles"] * c["ctx"] * bool(c.get("masked")), "flops": 4.0 * rows * c["ctx"]}
    return {"bytes": e * (2 * rows + 2 * kv * (c["prefix"] + c["tiles"] * c["own"])), "flops": 4.0 * rows * (c["prefix"] + c["own"])}


# ------------------------------------------------------------------------------------------------ 64-bit results
def _exact_rows(q, k, v):
    """softmax(q k^T / sqrt(d)) v of one head; q, k, v in 64 bits, no key: zeros."""
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    logits = (q / math.sqrt(q.shape[1])).mm(k.t())
    return torch.exp(logits - torch.logsumexp(logits, dim=1)[:, None]).mm(v)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "norm":
        total = s["x"].double()
        if c["residual"]:
            total += s["residual"].double()
        norm = (total.pow(2).sum(dim=2) / c["channels"] + 1e-6).sqrt()
        y = total / norm[:, :, None] * s["weight"].double()
        got = {"out": y, "sum": total} if c["residual"] else {"out": y}
        if c["out"] == "e4m3":   # the value that the 8 bits round, in units of the scale
            width = c["group"] or c["channels"]
            parts = y.unflatten(2, (c["channels"] // width, width))
            got["scale"] = torch.maximum(parts.amax(dim=3), -parts.amin(dim=3)) / E4M3_MAX
            got["out"] = (parts / got["scale"][..., None]).flatten(2)
        return got
    out = torch.empty(_queries_shape(c), dtype=torch.float64, device=DEV)

    def head_of(x, a):
        return (x[:, a] if c.get("token_major") else x[a]).double()

    for i in range(c["tiles"]):
        count = s["k"].shape[2 - bool(c.get("token_major"))] if s["len"] is None else int(s["len"][i])
        index = torch.arange(count, device=DEV)
        if s.get("mask") is not None:
            index = index[s["mask"][i, :count] != 0]
        for a in range(c["heads"]):
            b = a // (c["heads"] // c["kv_heads"])
            k, v = (head_of(s[key][i], b)[index] for key in ("k", "v"))
            if c["kind"] == "prefix":
                k, v = torch.cat([head_of(s["pk"], b), k]), torch.cat([head_of(s["pv"], b), v])
            o = _exact_rows(head_of(s["q"][i], a), k, v)
            if c.get("token_major"):
                out[i, :, a] = o
            else:
                out[i, a] = o
    return out
