"""References in 64 bits for the operators on the heads of a projection, with how far off a result may be.

Bounds count roundings: half a step of the result's type (``finfo.eps / 2`` relative to the value), ``n`` half steps of the type that
the arithmetic in between has (fp32, fp64 for fp64) for sums of ``n`` terms, and the angles' own error.
"""
import torch

from block_ref import F32, half_step, sequences

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


# ------------------------------------------------------------------------ cache in 8 bits ---

def e4m3(x):
    """The nearest value of e4m3 to one of at most 448, ties to even, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def quantised(x):
    """(values, scales) in 64 bits of rows (..., dim) in 64 bits.  A scale is rounded to fp32; a value is that of x over the scale before that."""
    top = x.abs().amax(-1)
    fine = torch.isfinite(top)
    top = torch.where(fine, top, torch.ones(())).clamp(min=2.0 ** -100)
    values = torch.where(fine[..., None], e4m3(torch.where(fine[..., None], x, torch.zeros((), dtype=x.dtype)) * 448.0 / top[..., None]), 0.0)
    return values, torch.where(fine, (top.float() / 448.0).double(), torch.nan)


def cache_rows(c, s, hk, count):
    """(values of keys, of values, scales of keys, of values) of the first `count` places of sequence s, in 64 bits."""
    place = torch.arange(count)
    page = c["table"].cpu()[s].long()[place // c["page"]].clamp(0, c["cache"].k.shape[0] - 1)
    at = place % c["page"]
    k, v = (t.cpu().double()[page, hk, at] for t in c["cache"][:2])
    ks, vs = (t.cpu().double()[page, hk, at] for t in c["cache"][2:])
    return k, v, ks, vs


def shaped_scores(qh, kh, scale, cap, slope, place, meet):
    """(scores, -inf where masked; tanh or None; how far off each may be) of queries at `place` of the keys' places."""
    d = qh.shape[1]
    x = scale * (qh @ kh.T)
    size = scale * (qh.abs() @ kh.abs().T)
    off = torch.zeros_like(x) + ((d + 16) * 2 * F32 * max(1.0, float(size[torch.isfinite(size)].max()) if size.numel() else 1.0))
    t = None
    if cap:
        t = torch.tanh(x / cap)
        x = cap * t
        off = off + 6 * F32 * cap
    if slope:
        bias = slope * (place[:, None] - torch.arange(kh.shape[0])[None]).abs()
        x = x - bias
        off = off + 4 * F32 * bias
    off = off + 2 * F32 * torch.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0).abs()
    return x.masked_fill(~meet, -torch.inf), t, off


def attend(x, off, v, size, dtype, lost=None):
    """(out, lse, bound, bound of lse) of scores x (rows, keys) over values v; size: |v|.  lost: per row and key, what the rounding of a
    weight leaves beside half a step of its own value."""
    step = half_step(dtype)
    if not x.shape[1]:
        z = torch.zeros((x.shape[0], v.shape[1]), dtype=torch.float64)
        return z, torch.full((x.shape[0],), -torch.inf, dtype=torch.float64), z, z[:, 0] if v.shape[1] else None
    lse = torch.logsumexp(x, 1)
    p = torch.where(x == -torch.inf, 0.0, torch.exp(x - lse[:, None]))
    out = _product(p, v)
    e = step + off + (x.shape[1] // 16 + 24) * F32
    far = _product(p * e, size) + _product(p * off, torch.ones_like(size)) * out.abs()
    if lost is not None:
        far = far + _product(lost(p), torch.ones_like(size))
    far = 1.05 * far + step * out.abs() + (2.0 ** -25 if dtype == torch.float16 else torch.finfo(dtype).tiny)
    return out, lse, far, 1.05 * (p * off).sum(1) + (x.shape[1] // 16 + 24) * F32 + 4 * F32 * torch.nan_to_num(lse, neginf=0.0).abs()


def _product(p, v):
    """p @ v where 0 times what is not finite is 0."""
    if bool(torch.isfinite(v).all()):
        return p @ v
    return torch.where(p[:, :, None] == 0, torch.zeros((), dtype=p.dtype), p[:, :, None] * v[None]).sum(1)


def cache_attention(c, causal=True, scale=None, cap=None, slopes=None, tree=None):
    """(out, lse, bound, bound of lse) of attention over a cache; rows of no sequence are NaN."""
    q = c["q"].double().cpu()
    t = c["q"].dtype
    n, heads, d = q.shape
    hk = c["cache"].k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, lse = torch.full(q.shape, torch.nan, dtype=torch.float64), torch.full(q.shape[:2], torch.nan, dtype=torch.float64)
    far, far_lse = torch.zeros_like(out), torch.zeros_like(lse)
    offsets, room = c["offsets"].tolist(), c["table"].shape[1] * c["page"]
    for s, length in enumerate(c["lengths"].tolist()):
        rows = slice(offsets[s], offsets[s + 1])
        nq, nk = rows.stop - rows.start, min(max(length, 0), room)
        first = max(length, 0) - nq                        # (also where the table has no room for it)
        place = torch.arange(nq) + first
        j = torch.arange(nk)
        meet = (j[None] <= place[:, None]) if causal else torch.ones(nq, nk, dtype=torch.bool)
        if tree is not None:
            b = j - first
            bits = tree.cpu()[rows]
            meet = (b < 0)[None] | ((b >= 0) & (b < 64))[None] & ((bits[:, None] >> b.clamp(0, 63)[None]) & 1).bool()
        for g in range(hk):
            k8, v8, ks, vs = cache_rows(c, s, g, nk)
            for h in range(g * heads // hk, (g + 1) * heads // hk):
                x, _, off = shaped_scores(q[rows, h], k8 * ks[:, None], scale, cap, 0.0 if slopes is None else float(slopes[h]), place, meet)

                def lost(p):                               # fp16: 2^-36 of the row's largest weight times scale, times the value
                    top = torch.nan_to_num(p * vs).amax(1, keepdim=True)
                    return 2.0 ** -36 * top * (meet.double() @ torch.nan_to_num(v8.abs()).amax(1, keepdim=True)) * torch.ones_like(p) / max(1, nk)

                out[rows, h], lse[rows, h], far[rows, h], f = attend(x, off, v8 * vs[:, None], (v8 * vs[:, None]).abs(), t,
                                                                     lost if t == torch.float16 else None)
                if f is not None:
                    far_lse[rows, h] = f
    return out, lse, far, far_lse


# ------------------------------------------------------------- attention with shaped scores ---

def _problems(c, causal, scale, cap, slopes, prefix):
    """Per sequence and head: (rows, keys, head, key head, q, k, v, scores, tanh, how far off scores are, which pairs meet)."""
    q, k, v = (c[n].double().cpu() for n in "qkv")
    group = q.shape[1] // k.shape[1]
    for s, (rows, keys) in enumerate(sequences(c["offsets"], c["key_offsets"], c["key_lengths"])):
        nq, nk = rows.stop - rows.start, keys.stop - keys.start
        place, j = torch.arange(nq) + nk - nq, torch.arange(nk)
        first = 0 if prefix is None else int(prefix[s])
        meet = (j[None] <= place[:, None]) | (j < first)[None] if causal else torch.ones(nq, nk, dtype=torch.bool)
        for h in range(q.shape[1]):
            qh, kh, vh = q[rows, h], k[keys, h // group], v[keys, h // group]
            x, t, off = shaped_scores(qh, kh, scale, cap, 0.0 if slopes is None else float(slopes[h]), place, meet)
            yield rows, keys, h, h // group, qh, kh, vh, x, t, off, meet


def shaped_attention(c, causal=True, scale=None, cap=None, slopes=None, prefix=None):
    """(out, lse, bound, bound of lse); rows of no sequence are NaN."""
    scale = c["q"].shape[2] ** -0.5 if scale is None else scale
    t = c["q"].dtype
    out, lse = torch.full(c["q"].shape, torch.nan, dtype=torch.float64), torch.full(c["q"].shape[:2], torch.nan, dtype=torch.float64)
    far, far_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for rows, _, h, _, _, _, vh, x, _, off, meet in _problems(c, causal, scale, cap, slopes, prefix):
        def lost(p):                                       # fp16: 2^-36 of the sum, times the value
            return 2.0 ** -36 * (meet.double() @ torch.nan_to_num(vh.abs()).amax(1, keepdim=True)) * torch.ones_like(p) / max(1, vh.shape[0])

        out[rows, h], lse[rows, h], far[rows, h], f = attend(x, off, vh, vh.abs(), t, lost if t == torch.float16 else None)
        if f is not None:
            far_lse[rows, h] = f
    return out, lse, far, far_lse


def shaped_attention_grad(c, out, lse, causal=True, scale=None, cap=None, slopes=None, prefix=None):
    """((dq, bound), (dk, bound), (dv, bound)) of the formula on these inputs; rows of no sequence are NaN."""
    scale = c["q"].shape[2] ** -0.5 if scale is None else scale
    t = c["q"].dtype
    step, tiny16 = half_step(t), 2.0 ** -25 if t == torch.float16 else torch.finfo(t).tiny
    dout, o, l = (x.double().cpu() for x in (c["dout"], out, lse))
    dq, dk, dv = (torch.full(c[n].shape, torch.nan, dtype=torch.float64) for n in "qkv")
    fq, fk, fv = (torch.zeros_like(x) for x in (dq, dk, dv))
    rounded = []
    for _, keys in sequences(c["offsets"], c["key_offsets"], c["key_lengths"]):
        dk[keys], dv[keys] = 0.0, 0.0
    for rows, keys, h, g, qh, kh, vh, x, tanh, off, meet in _problems(c, causal, scale, cap, slopes, prefix):
        if not kh.shape[0]:
            dq[rows, h] = 0.0
            continue
        dy = dout[rows, h]
        p = torch.where(meet, torch.exp(torch.where(meet, x, 0.0) - l[rows, h][:, None]), 0.0)
        delta = (dy * o[rows, h]).sum(1)[:, None]
        dp = dy @ vh.T
        turn = 1.0 if tanh is None else 1.0 - tanh.square()
        ds = torch.where(meet, scale * p * (dp - delta) * turn, 0.0)
        more = (max(x.shape) // 16 + 24) * F32
        e = (qh.shape[1] + 8) * 2 * F32 * (dy.abs() @ vh.abs().T + (dy * o[rows, h]).abs().sum(1)[:, None])
        fds = 1.05 * ((step + off + more) * ds.abs() + scale * p * e)
        if cap:                                            # the tanh is off by some 2^-23, its derivative by twice that, and by the score's error
            fds = fds + scale * p * (dp - delta).abs() * (16 * F32 + 2 * off / cap)
        sub = 2.0 ** -36 if t == torch.float16 else 0.0    # fp16: of the largest of the row (dq), of the rows of all heads of the key head (dk)
        rounded.append((keys, g, ds.abs().amax() if ds.numel() else 0.0, meet.double().T @ qh.abs()))
        dq[rows, h] = _product(ds, kh)
        fq[rows, h] = 1.01 * step * dq[rows, h].abs() + _product(fds + sub * ds.abs().amax(1, keepdim=True) * meet, kh.abs()) + tiny16
        dk[keys, g] += _product(ds.T, qh)
        fk[keys, g] += _product(fds.T, qh.abs())
        dv[keys, g] += _product(p.T, dy)
        fv[keys, g] += _product((1.05 * (step + off + more) * p + (2.0 ** -40 if sub else 0.0) * meet).T, dy.abs())
    for keys, g, _, size in rounded if t == torch.float16 else []:
        fk[keys, g] += 2.0 ** -36 * max(float(r[2]) for r in rounded if r[:2] == (keys, g)) * size
    return (dq, fq), (dk, fk + 1.01 * step * dk.abs() + tiny16), (dv, fv + 1.01 * step * dv.abs() + tiny16)
