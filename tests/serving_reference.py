"""Plain 64-bit forms of the served attention block's operators, for the tests: straight from the formulas in include/gc.h,
one row, group or head at a time, on whatever device their inputs live."""
import math

import torch


def rope(x, weight, positions, inv_freq, norm, eps, interleaved, factor):
    """x [T, H, D] -> (result, |a| + |b| of every element's pair: what errors of cos / sin scale with)."""
    y = x.double()
    if norm:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double()
    half = inv_freq.numel()
    phi = positions.double()[:, None, None] * inv_freq.double()
    c, s = torch.cos(phi) * factor, torch.sin(phi) * factor
    out, size = y.clone(), y.abs()
    if half:
        at = torch.arange(half, device=x.device)
        ia, ib = (2 * at, 2 * at + 1) if interleaved else (at, at + half)
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, size


def bf16_floor(x):
    """The largest bf16 <= x (64 bits): eight significant bits, the last place never below the smallest bf16 step."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), torch.clamp(e - 8, min=-133))
    return torch.floor(x / step) * step


def quantise(x, group):
    """x [..., D] -> (codes [..., D], lo, scale [..., D / group]) in 64 bits, on the exact quotients."""
    g = x.double().unflatten(-1, (-1, group))
    lo = bf16_floor(g.amin(-1))
    fifteen = torch.full_like(lo, 15.0)
    scale = -bf16_floor(-((g.amax(-1) - lo) / fifteen))
    unit = torch.where(scale > 0, scale, torch.ones_like(scale))
    code = torch.where(scale[..., None] > 0, ((g - lo[..., None]) / unit[..., None]).round(), torch.zeros_like(g)).clamp(0, 15)
    return code.flatten(-2), lo, scale


def values(codes, params):
    """The values a cache holds: codes u8 [..., D / 2], params [..., groups, 2] -> (values, lo of each) [..., D] in 64 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
    p = params.double()
    c = c.unflatten(-1, (p.shape[-2], -1))
    lo = p[..., 0, None].expand_as(c)
    return (lo + c * p[..., 1, None]).flatten(-2), lo.flatten(-2)


def head(q, k, v, limits, scale):
    """softmax(scale q k^T) v of one head; row i sees the first limits[i] keys, zero where there is none.  Masked keys and
    values are never touched.  Also sum p |v| / sum p."""
    o = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64, device=q.device)
    size = torch.zeros_like(o)
    for i in range(q.shape[0]):
        n = int(limits[i])
        if n > 0:
            p = torch.softmax(scale * (k[:n] @ q[i]), 0)
            o[i], size[i] = p @ v[:n], p @ v[:n].abs()
    return o, size


def head_all(q, k, v, limits, scale):
    """The same with all rows at once, for longer sequences of finite numbers."""
    s = scale * (q @ k.T)
    s = s.masked_fill(torch.arange(k.shape[0], device=q.device) >= limits[:, None], -math.inf)
    p = torch.nan_to_num(torch.softmax(s, -1))
    return p @ v, p @ v.abs()
