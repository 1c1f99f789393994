"""References in 64 bits for the operators of a transformer block, with how far off a result may be.

A result's bound counts roundings: half a step of the result's type (``finfo.eps / 2`` relative to the value), half a step of
the type for every operand that the matrix units take rounded, and ``n`` half steps of fp32 for sums in fp32.
"""
import math

import torch

F32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def within(got, ref, bound, what):
    got, ref, bound = got.detach().double().cpu(), ref.detach().double().cpu(), bound.detach().double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = (got == ref) | (got.isnan() & ref.isnan())
    far = ~same & ~((got - ref).abs() <= bound)
    if far.any():
        i = tuple(far.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d values off, first at %s: got %r, reference %r, bound %.3e" %
                             (what, int(far.sum()), far.numel(), i, float(got[i]), float(ref[i]), float(bound[i])))


# ------------------------------------------------------------------------------ norms ---

def norm(v, weight, kind, eps):
    w, b = weight if isinstance(weight, tuple) else (weight, None)
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    n = v / (v.square().mean(1, keepdim=True) + eps).sqrt()
    return n * w if b is None else n * w + b


def block(x, z, gate, scale, post, pre, kind, eps):
    """(h, y) from float64 tensors"""
    h = x
    if z is not None:
        u = z if post is None else norm(z, post, kind, eps)
        if gate is not None:
            u = u * (gate[1][:, None] if gate[0] == "colvec" else gate[1])
        h = x + scale * u
    return h, None if pre is None else norm(h, pre, kind, eps)


# -------------------------------------------------------------------------- attention ---

def sequences(offsets, key_offsets, key_lengths):
    o = offsets.tolist()
    k = o if key_offsets is None else key_offsets.tolist()
    for s in range(len(o) - 1):
        n = k[s + 1] - k[s]
        yield slice(o[s], o[s + 1]), slice(k[s], k[s] + (n if key_lengths is None else min(n, int(key_lengths[s]))))


def _scores(q, k, scale, causal):
    n, m = q.shape[0], k.shape[0]
    s = scale * (q @ k.T)
    if causal:
        s = s.masked_fill(torch.arange(m)[None, :] > torch.arange(n)[:, None] + (m - n), -math.inf)
    return s


def _spread(q, k, scale):
    """How far off exp(S - max) may be, relative to itself: fp32 sums over dim, times the scale."""
    d = q.shape[1]
    top = float((scale * (q.abs() @ k.abs().T)).max()) if q.shape[0] and k.shape[0] else 0.0
    return (d + 16) * 2 * F32 * max(1.0, top)


def attention(q, k, v, offsets, key_offsets=None, key_lengths=None, causal=True, scale=None, skip=None):
    """(out, lse, bound of out, bound of lse); rows of no sequence are NaN.  Masked keys are left out, not multiplied with 0."""
    t, step = q.dtype, half_step(q.dtype)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    group = q.shape[1] // k.shape[1]
    out, lse = torch.full(q.shape, math.nan, dtype=torch.float64), torch.full(q.shape[:2], math.nan, dtype=torch.float64)
    far, far_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for qs, ks in sequences(offsets, key_offsets, key_lengths):
        for h in range(q.shape[1]):
            qh, kh, vh = q[qs, h], k[ks, h // group], v[ks, h // group]
            s = _scores(qh, kh, scale, causal)
            l = torch.logsumexp(s, 1) if s.shape[1] else torch.full((s.shape[0],), -math.inf, dtype=torch.float64)
            p = torch.where(s == -math.inf, 0.0, torch.exp(s - l[:, None])) if s.numel() else torch.zeros_like(s)
            o = product(p, vh)
            off = _spread(qh, kh, scale)
            out[qs, h], lse[qs, h] = o, l
            far[qs, h] = step * o.abs() + 1.05 * (step + off) * product(p, vh.abs()) + torch.finfo(t).tiny
            far_lse[qs, h] = off + 4 * F32 * l.abs()
    return out, lse, far, far_lse


def product(p, v):
    """p @ v where 0 * NaN and 0 * inf are 0 (p is 0 for masked keys only, or where it is too small for 64 bits)."""
    if bool(torch.isfinite(v).all()):
        return p @ v
    return torch.where(p[:, :, None] == 0, torch.zeros((), dtype=p.dtype), p[:, :, None] * v[None]).sum(1)


def attention_grad(dout, q, k, v, out, lse, offsets, key_offsets=None, key_lengths=None, causal=True, scale=None):
    """((dq, bound), (dk, bound), (dv, bound)) of the formula on these inputs; rows of no sequence are NaN."""
    step = half_step(q.dtype)
    tiny = torch.finfo(q.dtype).tiny
    scale = q.shape[2] ** -0.5 if scale is None else scale
    dout, q, k, v, out, lse = (t.double().cpu() for t in (dout, q, k, v, out, lse))
    group, d = q.shape[1] // k.shape[1], q.shape[2]
    dq, dk, dv = (torch.full(t.shape, math.nan, dtype=torch.float64) for t in (q, k, v))
    fq, fk, fv = torch.zeros_like(dq), torch.zeros_like(dk), torch.zeros_like(dv)
    for qs, ks in sequences(offsets, key_offsets, key_lengths):
        dk[ks], dv[ks] = 0.0, 0.0
        for h in range(q.shape[1]):
            qh, kh, vh, g, o = q[qs, h], k[ks, h // group], v[ks, h // group], dout[qs, h], out[qs, h]
            if not kh.shape[0]:
                dq[qs, h] = 0.0
                continue
            s = _scores(qh, kh, scale, causal)
            p = torch.where(s == -math.inf, 0.0, torch.exp(s - lse[qs, h][:, None]))
            delta, dp = (g * o).sum(1)[:, None], g @ vh.T
            seen = s != -math.inf
            ds = torch.where(seen, scale * p * (dp - delta), 0.0)
            off = _spread(qh, kh, scale)
            e = (d + 8) * 2 * F32 * (g.abs() @ vh.abs().T + (g * o).abs().sum(1)[:, None])
            fds = 1.05 * ((step + off) * ds.abs() + scale * p * e)
            dq[qs, h] = product(ds, kh)
            fq[qs, h] = step * dq[qs, h].abs() + product(fds, kh.abs()) + tiny
            dk[ks, h // group] += product(ds.T, qh)
            fk[ks, h // group] += product(fds.T, qh.abs())
            dv[ks, h // group] += product(p.T, g)
            fv[ks, h // group] += 1.05 * (step + off) * product(p.T, g.abs())
    return (dq, fq), (dk, fk + step * dk.abs() + tiny), (dv, fv + step * dv.abs() + tiny)
