"""Plain 64-bit forms of rotary positions, gated norms and 8-bit integer linear layers, and how far a kernel may be from them (not a test module).

Half a step of the types (torch.finfo(t).eps / 2, relative): fp32 2^-24, bf16 2^-8, e4m3 2^-4.
"""
import math

import torch

U32, U16, U8 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4
UNIT = {"f32": U32, "bf16": U16}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
TINY = 1e-30
# Sums of a row: a lane adds up to 32 products (one rounding more each) in order, then at most 10 joins of lanes and wavefronts.
SUM = 48 * U32


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def centred64(x, kind, eps):
    """(z, sigma) of rows in fp64."""
    if kind == "none":
        return x, torch.ones_like(x[:, :1])
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    sigma = (x.square().mean(dim=1, keepdim=True) + eps).sqrt()
    return x / sigma, sigma


def centred_error(z, sigma, err, kind):
    """Error of z = centred64(v) where v is off by err.  The norm's factor: half the relative error of a mean of squares, the root and two products.
    The mean of the layer norm: SUM of mean|v - mean|, which is below sigma, and the roundings of the two differences."""
    if kind == "none":
        return err
    own = (SUM / 2 + 8 * U32) * z.abs()
    if kind == "layer":
        own = own + SUM + 4 * U32 * z.abs()
        err = err + err.mean(dim=1, keepdim=True)
    return own + (err + z.abs() * err.square().mean(dim=1, keepdim=True).sqrt()) / sigma


def per_row(v, rows, mod_rows):
    v = v.double()
    return v[torch.arange(rows) // mod_rows] if mod_rows else v[:1].expand(rows, -1)


def gated64(x, residual, gate, post_weight, weight, scale, shift, norm, post, residual_scale, mod_rows, eps):
    """(s, error of s, y, error of y) of one tile; all tensors on the CPU, residual .. shift or None."""
    rows = x.shape[0]
    z, sigma = centred64(x.double(), post, eps)
    err = centred_error(z, sigma, torch.zeros_like(z), post)
    for w in (None if post_weight is None else post_weight.double(), None if gate is None else per_row(gate, rows, mod_rows)):
        if w is not None:
            z = z * w
            err = err * w.abs() + U32 * z.abs()
    if residual is not None:
        r = float(torch.tensor(residual_scale, dtype=torch.float32)) * residual.double()
        s = z + r
        err = err + U32 * s.abs()
    else:
        s = z
    y, sigma = centred64(s, norm, eps)
    err_y = centred_error(y, sigma, err, norm)
    for w in (None if weight is None else weight.double(), None if scale is None else 1 + per_row(scale, rows, mod_rows)):
        if w is not None:
            y = y * w
            err_y = err_y * w.abs() + 2 * U32 * y.abs()
    if shift is not None:
        y = y + per_row(shift, rows, mod_rows)
        err_y = err_y + U32 * y.abs()
    return s, err, y, err_y


def rotary64(x, freq, coords, axes, layout, weight=None, eps=1e-6):
    """(result, error) of x [tokens][heads][d] in fp64, coords [tokens][3]."""
    axis_of = torch.repeat_interleave(torch.arange(3), torch.tensor([n // 2 for n in axes]))
    angle = coords.double()[:, axis_of] * freq
    cos, sin = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
    d, turned = x.shape[-1], sum(axes)
    x = x.double()
    err = torch.zeros_like(x)
    if weight is not None:
        x = x / (x.square().mean(dim=-1, keepdim=True) + eps).sqrt() * weight.double()
        err = (SUM / 2 + 10 * U32) * x.abs()
    y, tol = x.clone(), err.clone()
    pick = (slice(0, turned // 2), slice(turned // 2, turned)) if layout == "half" else (slice(0, turned, 2), slice(1, turned, 2))
    a, b = x[..., pick[0]], x[..., pick[1]]
    y[..., pick[0]], y[..., pick[1]] = a * cos - b * sin, b * cos + a * sin
    both = err[..., pick[0]] + err[..., pick[1]] + (2.0 ** -21 + 3 * U32) * (a.abs() + b.abs())
    tol[..., pick[0]], tol[..., pick[1]] = both, both
    assert d >= turned
    return y, tol


def linear64(x, x_scale, w, w_scale, bias, gelu):
    """(result, error) of one tile in fp64: the sum is exact, then it is rounded, multiplied and added to (3 roundings)."""
    p = (x.double() @ w.double().t()) * x_scale.double()[:, None] * w_scale.double()
    v = p if bias is None else p + bias.double()
    err = 3 * U32 * p.abs() + U32 * v.abs()
    if not gelu:
        return v, err
    u = math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    y = v * torch.sigmoid(2 * u)
    # slope of GELU below 1.13; the exponent's argument is off by 5 roundings, the exponential, sum, reciprocal and product by 8
    return y, 1.13 * err + (10 * u.abs() + 8) * U32 * y.abs()


def check(got, ref, tol, dtype):
    u = UNIT[dtype]
    off = (got.cpu().double() - ref).abs()
    assert bool((off <= tol + u * (ref.abs() + tol) + TINY).all()), float((off - tol - u * ref.abs()).max())


def check_eight(got, scale, ref, tol, kind, group):
    """got: 8-bit rows, scale: [rows][blocks]."""
    rows, c = ref.shape
    blocks, t = ref.view(rows, -1, group or c), tol.view(rows, -1, group or c)
    top = 127.0 if kind == "int8" else 448.0
    sc = scale.cpu().double().view(rows, -1)
    most = blocks.abs().amax(dim=-1)
    assert bool(((sc * top - most).abs() <= t.amax(dim=-1) + 4 * U32 * most + TINY).all())
    deq = got.cpu().float().double().view(blocks.shape) * sc[..., None]
    step = 0.5 * sc[..., None] if kind == "int8" else U8 * blocks.abs() + 2.0 ** -10 * sc[..., None]
    assert bool(((deq - blocks).abs() <= t * (1 + U8) + 8 * U32 * blocks.abs() + step * (1 + 8 * U32) + TINY).all())
