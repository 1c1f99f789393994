"""References in 64 bits for the operators on the heads of a projection, with how far off a result may be.

Bounds count roundings: half a step of the result's type (``finfo.eps / 2`` relative to the value), ``n`` half steps of the type that
the arithmetic in between has (fp32, fp64 for fp64) for sums of ``n`` terms, and the angles' own error.
"""
import torch

from block_ref import F32, half_step

F64 = 2.0 ** -53


def inner(dtype):
    """Half a step of the arithmetic in between."""
    return F64 if dtype == torch.float64 else F32


# ------------------------------------------------------------- norms and rotary positions ---

def angles(positions, freqs, sections):
    """(tokens, pairs) in 64 bits"""
    positions, freqs = positions.cpu(), freqs.cpu()
    p = positions.view(1, -1) if positions.dim() == 1 else positions
    sections = (freqs.numel(),) if sections is None else sections
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    return p.double()[axis].T * freqs


def split(x, half, pairs):
    """(first of every pair, second, the rest)"""
    front = x[..., :2 * half]
    a, b = (front[..., :half], front[..., half:]) if pairs == "halves" else (front[..., 0::2], front[..., 1::2])
    return a, b, x[..., 2 * half:]


def joined(a, b, rest, pairs):
    front = torch.cat([a, b], -1) if pairs == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([front, rest], -1)


def rotary(x, weight, angle, pairs, eps):
    """Result in 64 bits of one tensor (tokens, heads, dim) in 64 bits."""
    y = x if weight is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight
    a, b, rest = split(y, angle.shape[1], pairs)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    return joined(a * c - b * s, a * s + b * c, rest, pairs)


def rotary_bound(x, weight, angle, pairs, eps, dtype):
    """How far off the result of type dtype may be."""
    f = inner(dtype)
    y = x.abs() if weight is None else (x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight).abs()
    norm = 0 if weight is None else (x.shape[-1] / 2 + 16) * f
    a, b, rest = split(y, angle.shape[1], pairs)
    both = (a + b) * (norm + turn_error(angle, dtype) + 4 * f)
    return half_step(dtype) * 1.01 * rotary(x, weight, angle, pairs, eps).abs() + joined(both, both, rest * (norm + 2 * f), pairs) + tiny(dtype)


def turn_error(angle, dtype):
    """Of cos and sin: a few steps of their own, and the angle's when whole turns are taken off it."""
    return (8 * inner(dtype) + angle.abs() * (2.0 ** -52 if dtype == torch.float64 else 2.0 ** -51))[:, None]


def tiny(dtype):
    return torch.finfo(dtype).tiny * (half_step(dtype) if dtype in (torch.float32, torch.float64) else 1.0) if dtype != torch.float16 else 2.0 ** -25


def rotary_grad(dy, x, weight, angle, pairs, eps, dtype):
    """((dx, bound), (dweight, bound) or None)"""
    f, dim = inner(dtype), dy.shape[-1]
    a, b, rest = split(dy, angle.shape[1], pairs)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    g = joined(a * c + b * s, b * c - a * s, rest, pairs)
    size = (a.abs() + b.abs())
    far = joined(size * (turn_error(angle, dtype) + 4 * f), size * (turn_error(angle, dtype) + 4 * f), torch.zeros_like(rest), pairs)
    if weight is None:
        return (g, 1.01 * half_step(dtype) * g.abs() + far + tiny(dtype)), None
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    gw = g * weight
    mean = (gw * x).mean(-1, keepdim=True) * r * r
    dx = r * (gw - x * mean)
    size = r * (gw.abs() + x.abs() * (gw * x).abs().mean(-1, keepdim=True) * r * r)
    more = r * (far * weight.abs() + x.abs() * (far * weight.abs() * x.abs()).mean(-1, keepdim=True) * r * r)
    dw = (g * x * r).sum((0, 1))
    # adds in a row: a lane's rows, a block's lanes, the blocks
    heads, tokens = dy.shape[1], dy.shape[0]
    chain = min(heads * tokens, heads * 4 * (tokens // 4096 + 1) + 340) + dim / 2 + 24
    fw = ((far + chain * f * g.abs()) * x.abs() * r).sum((0, 1))
    return (dx, 1.01 * half_step(dtype) * dx.abs() + (2 * dim + 48) * f * size + 1.01 * more + tiny(dtype)), \
        (dw, 1.01 * half_step(dtype) * dw.abs() + 1.01 * fw + tiny(dtype))
