"""Operators of a transformer block: thin wrappers with the names of the C entry points (argument marshalling only).

Workspaces are torch tensors made on the call's stream, so a call that is captured into a HIP graph keeps its own in the
graph's memory pool, and two graphs or streams share none.
"""
import ctypes
from collections import namedtuple
from contextlib import contextmanager

import torch

from . import _lib as L
from .api import SIDE, _check, _raw_stream

NORM = {"rms": 0, "layer": 1}
DTYPE = {torch.float64: 0, torch.float32: 1, torch.bfloat16: 2, torch.float16: 3}

BlockGrads = namedtuple("BlockGrads", "dx dz dgate dpost dpost_bias dpre dpre_bias")
"""Gradients of fuse_block_norm; None where the call had no such input."""


def _handle(device, stream):
    """The stream's handle where a call runs as things are: on the current device and its current stream.  None: see _on."""
    if device.type != "cuda":
        raise ValueError("tensors must be CUDA (HIP) tensors, got device %s" % device)
    if stream is None and _raw_stream is not None and device.index == torch.cuda.current_device():
        return _raw_stream(device.index)
    return None


@contextmanager
def _on(device, stream):
    """The device, and the stream on it (default: its current one), that a call runs on; yields the stream's handle.
    Allocations inside belong to that stream."""
    if stream is not None and not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    if stream is not None and stream.device != device:
        raise ValueError("the stream is on %s, the tensors are on %s" % (stream.device, device))
    with torch.cuda.device(device):
        if stream is None:
            stream = torch.cuda.current_stream(device)
        with torch.cuda.stream(stream):
            yield stream.cuda_stream


def _run(device, stream, call):
    """call(handle) on the device and stream."""
    handle = _handle(device, stream)
    if handle is not None:
        return call(handle)
    with _on(device, stream) as handle:
        return call(handle)


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def _like(t, x, what):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % what)
    if t.dtype is not x.dtype:
        raise TypeError("%s is %s, not %s" % (what, t.dtype, x.dtype))
    if t.device != x.device:
        raise ValueError("%s is on %s, not on %s" % (what, t.device, x.device))
    return t


def _dtype(x, what):
    if not isinstance(x, torch.Tensor) or x.dtype not in DTYPE:
        raise TypeError("%s must be a float64, float32, bfloat16 or float16 tensor" % what)
    return DTYPE[x.dtype]


# ------------------------------------------------------------------------------ norms ---

def _rows_of(t, x, what):
    """Pointer and leading dimension of a matrix of x's shape with unit column stride."""
    if t is not x:
        _like(t, x, what)
        if t.shape != x.shape:
            raise ValueError("%s has shape %s, not %s" % (what, tuple(t.shape), tuple(x.shape)))
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s needs unit column stride" % what)
    return t.data_ptr(), ld if rows > 1 else cols


def _vector(t, x, count, what):
    _like(t, x, what)
    if t.dim() != 1 or t.numel() != count or (count > 1 and t.stride(0) != 1):
        raise ValueError("%s must be a contiguous vector of %d values" % (what, count))
    return t.data_ptr()


def _weights(p):
    return (None, None) if p is None else p if isinstance(p, tuple) else (p, None)


def _block(x, z, gate, scale, post, pre, kind, eps, what):
    """(descriptor, gate's kind and tensor) of a block around matrices of x's shape and type."""
    dtype = _dtype(x, what)
    if x.dim() != 2:
        raise ValueError("%s must be a matrix" % what)
    if kind not in NORM:
        raise ValueError("kind is 'rms' or 'layer', not %r" % (kind,))
    rows, cols = x.shape
    zp, z_ld = (None, 0) if z is None else _rows_of(z, x, "z")
    (post_w, post_b), (pre_w, pre_b) = _weights(post), _weights(pre)
    post_wp = None if post_w is None else _vector(post_w, x, cols, "post weight")
    post_bp = None if post_b is None else _vector(post_b, x, cols, "post bias")
    pre_wp = None if pre_w is None else _vector(pre_w, x, cols, "pre weight")
    pre_bp = None if pre_b is None else _vector(pre_b, x, cols, "pre bias")
    gk, gt = (None, None) if gate is None else gate
    code, gp, g_ld = -1, None, 0
    if gk is not None:
        if gk not in ("rowvec", "colvec", "matrix"):
            raise ValueError("a gate is ('rowvec' | 'colvec' | 'matrix', tensor), not %r" % (gk,))
        code = SIDE[gk]
        if gk == "rowvec":
            gp = _vector(gt, x, cols, "gate")
        elif gk == "matrix":
            gp, g_ld = _rows_of(gt, x, "gate")
        else:
            _like(gt, x, "gate")
            if gt.dim() != 1 or gt.numel() != rows:
                raise ValueError("gate must be a vector of %d values" % rows)
            gp, g_ld = gt.data_ptr(), gt.stride(0) if rows > 1 else 1
        if not gt.numel():
            gp = x.data_ptr() or 16              # (no rows: never read)
    b = L.Block(dtype, NORM[kind], rows, cols, eps, scale, zp, z_ld, post_wp, post_bp, pre_wp, pre_bp, code, gp, g_ld)
    return b, gk, gt


def fuse_block_norm(x, z=None, gate=None, scale=1.0, post=None, pre=None, kind="rms", eps=1e-6, h=None, y=None, stream=None):
    """C: fuse_block_norm.  h = x + scale * gate * N_post(z), y = N_pre(h); returns (h, y).

    x, z: (rows, cols) on the GPU.  post, pre: weight, or (weight, bias) for kind="layer", of the norm after the block and of the
    one before the next; None: no such norm (then y is None, respectively z is added as it is).  gate: ("rowvec" | "colvec" |
    "matrix", tensor).  h, y: tensors to write to; h may be x.  Without z, h is x itself."""
    b, gk, gt = _block(x, z, gate, scale, post, pre, kind, eps, "x")
    if z is None and h is not None:
        raise ValueError("h needs the block's result z: without one it is x")
    if pre is None and y is not None:
        raise ValueError("y needs the norm that makes it: pre is None")
    xp, x_ld = _rows_of(x, x, "x")

    def call(handle):
        rh, ry, hp, yp = h, y, None, None
        h_ld = y_ld = b.cols
        if h is not None:
            hp, h_ld = _rows_of(h, x, "h")
        elif z is not None:
            rh = torch.empty_like(x, memory_format=torch.contiguous_format)
            hp = rh.data_ptr()
        if y is not None:
            yp, y_ld = _rows_of(y, x, "y")
        elif pre is not None:
            ry = torch.empty_like(x, memory_format=torch.contiguous_format)
            yp = ry.data_ptr()
        if b.rows and b.cols:
            _check(L.load().fuse_block_norm(b, xp, x_ld, hp, h_ld, yp, y_ld, handle))
        return x if rh is None else rh, ry

    return _run(x.device, stream, call)


def fuse_block_norm_backward(dh, dy, h, z=None, gate=None, scale=1.0, post=None, pre=None, kind="rms", eps=1e-6, stream=None):
    """C: fuse_block_norm_backward.  Gradients of fuse_block_norm from those of its results (one of them may be None: zero),
    its h (x where there was no z) and its other inputs: a BlockGrads."""
    like = h if h is not None else dh
    b, gk, gt = _block(like, z, gate, scale, post, pre, kind, eps, "h")
    (post_w, post_b), (pre_w, pre_b) = _weights(post), _weights(pre)
    lib = L.load()

    def new(t):
        return None if t is None else torch.empty_like(t, memory_format=torch.contiguous_format)

    def call(handle):
        got = BlockGrads(new(like), new(z), new(gt), new(post_w), new(post_b), new(pre_w), new(pre_b))
        if like.numel() == 0:
            for t in got:
                if t is not None:
                    t.zero_()
            return got
        cols = like.shape[1]
        dx, dz, dgate, dpost, dpost_bias, dpre, dpre_bias = [t.data_ptr() if t is not None else None for t in got]
        g = L.BlockGrads(dx, cols, dz, cols, dgate, cols if gk == "matrix" else 1, dpost, dpost_bias, dpre, dpre_bias)
        ws = _workspace(lib.fuse_block_norm_backward_bytes(b), like.device)
        args = []
        for t, what in ((dh, "dh"), (dy, "dy"), (h, "h")):
            args += _rows_of(t, like, what) if t is not None else (None, 0)
        _check(lib.fuse_block_norm_backward(b, *args, g, ws.data_ptr(), ws.numel(), handle))
        return got

    return _run(like.device, stream, call)


# -------------------------------------------------------------------------- attention ---

def _heads_of(t, like, what, tokens=None, heads=None):
    """(pointer, stride between tokens, stride between heads) of a (tokens, heads, dim) tensor with unit stride along dim."""
    if t is not like:
        _like(t, like, what)
    shape = t.shape
    if len(shape) != 3 or shape[2] != like.shape[2]:
        raise ValueError("%s must be (tokens, heads, %d)" % (what, like.shape[-1]))
    n, h, dim = shape
    if (tokens is not None and n != tokens) or (heads is not None and h != heads):
        raise ValueError("%s has shape %s, not (%s, %s, %d)" % (what, tuple(shape), tokens, heads, dim))
    token, head, step = t.stride()
    if step != 1 and dim > 1:
        raise ValueError("%s needs unit stride along dim" % what)
    return t.data_ptr(), token if n > 1 else dim * h, head if h > 1 else dim


def _places(t, like, device, count, what):
    if t.dtype is not like.dtype:
        raise TypeError("%s must be int32 or int64, like offsets" % what)
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (what, t.device, device))
    if t.dim() != 1 or t.numel() != count or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d values" % (what, count))
    return t.data_ptr()


def _row(t, like, dtype, count, what):
    """Pointer of a contiguous vector of `count` values of a type, on like's device."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        raise TypeError("%s must be a %s tensor" % (what, dtype))
    if t.device != like.device:
        raise ValueError("%s is on %s, not on %s" % (what, t.device, like.device))
    if t.dim() != 1 or t.numel() != count or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d values" % (what, count))
    return t.data_ptr()


def _cap(cap):
    """0: none"""
    if cap is not None and not cap > 0.0:
        raise ValueError("cap must be positive, or None for no cap")
    return 0.0 if cap is None else cap


def _attn(q, k, v, offsets, key_offsets, key_lengths, causal, scale):
    dtype = _dtype(q, "q")
    qs, ks = q.shape, k.shape
    if len(qs) != 3 or len(ks) != 3 or qs[1] < 1 or ks[1] < 1 or qs[2] < 1:
        raise ValueError("q, k and v must be (tokens, heads, dim)")
    qp, q_token, q_head = _heads_of(q, q, "q")
    kp, k_token, k_head = _heads_of(k, q, "k")
    vp, v_token, v_head = _heads_of(v, q, "v", ks[0], ks[1])
    if offsets is None or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets must be a vector of the number of sequences + 1 values")
    if offsets.dtype is not torch.int32 and offsets.dtype is not torch.int64:
        raise TypeError("offsets must be int32 or int64")
    if key_lengths is not None and key_offsets is None:
        raise ValueError("key_lengths needs key_offsets")
    device, seqs = q.device, offsets.numel() - 1
    qo = _places(offsets, offsets, device, seqs + 1, "offsets")
    ko = None if key_offsets is None else _places(key_offsets, offsets, device, seqs + 1, "key_offsets")
    kl = None if key_lengths is None else _places(key_lengths, offsets, device, seqs, "key_lengths")
    return L.Attn(dtype, qs[1], ks[1], qs[2], 1 if causal else 0, 1 if offsets.dtype is torch.int64 else 0, qs[0], ks[0], seqs, qo, ko, kl,
                  qs[2] ** -0.5 if scale is None else scale, qp, kp, vp, q_token, q_head, k_token, k_head, v_token, v_head)


def _shape(f, q, offsets, causal, cap, slopes, prefix):
    """What is done to the scores; None: nothing."""
    if cap is None and slopes is None and prefix is None:
        return None
    if prefix is not None and not causal:
        raise ValueError("a prefix goes with causal: without it all queries see all keys")
    return L.AttnShape(_cap(cap), None if slopes is None else _row(slopes, q, torch.float32, f.heads, "slopes"),
                       None if prefix is None else _places(prefix, offsets, q.device, f.seqs, "prefix"))


def fuse_attention(q, k, v, offsets, key_offsets=None, key_lengths=None, causal=True, scale=None, out=None, lse=None, stream=None, cap=None,
                   slopes=None, prefix=None):
    """C: fuse_attention, fuse_attention_shaped.  softmax(scale * q k^T + mask) v for packed sequences; returns (out, lse).

    q: (tokens, heads, dim), k and v: (key tokens, key heads, dim), bfloat16 or float16, heads a multiple of key heads; parts of
    one projection can be passed as they are.  offsets: the sequences' first queries and the end of the last one; key_offsets likewise
    for the keys (None: the same), with key_lengths only so many keys from each sequence's first one on (a cache with room).
    causal: the last query sees all keys, the one before it all but the last, and so on.  scale: None is 1 / sqrt(dim).  lse:
    (tokens, heads) float32.  Rows that belong to no sequence are not written: in results made here they hold anything (NaN
    among it: a padded batch whose other rows go on into sums over all rows takes out=torch.zeros_like(q)).
    cap: scores become cap * tanh(score / cap).  slopes: (heads,) float32, slopes[h] * |distance| is taken off the scores, in places among the
    keys.  prefix: a length per sequence, like offsets; all its queries see so many of its first keys (with causal)."""
    f = _attn(q, k, v, offsets, key_offsets, key_lengths, causal, scale)
    shape = _shape(f, q, offsets, causal, cap, slopes, prefix)
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.device != q.device):
        raise ValueError("lse must be a contiguous float32 tensor of shape %s on %s" % (tuple(q.shape[:2]), q.device))
    lib = L.load()

    def call(handle):
        n, heads, dim = q.shape
        l = torch.empty((n, heads), dtype=torch.float32, device=q.device) if lse is None else lse
        if out is None:
            o = torch.empty_like(q, memory_format=torch.contiguous_format)
            op, o_token, o_head = o.data_ptr(), heads * dim, dim
        else:
            o = out
            op, o_token, o_head = _heads_of(o, q, "out", n, heads)
        nbytes = lib.fuse_attention_bytes(f)
        ws = _workspace(nbytes, q.device) if nbytes else None
        args = (op, o_token, o_head, l.data_ptr(), ws.data_ptr() if nbytes else None, nbytes, handle)
        _check(lib.fuse_attention(f, *args) if shape is None else lib.fuse_attention_shaped(f, shape, *args))
        return o, l

    return _run(q.device, stream, call)


def fuse_attention_backward(dout, q, k, v, out, lse, offsets, key_offsets=None, key_lengths=None, causal=True, scale=None,
                            dq=None, dk=None, dv=None, stream=None, cap=None, slopes=None, prefix=None):
    """C: fuse_attention_backward, fuse_attention_shaped_backward.  Gradients (dq, dk, dv) of fuse_attention's out, given its results and its
    other arguments; slopes are constants.

    dq, dk, dv: tensors to write to.  Rows that belong to no sequence (before the first and behind the last one, and behind a sequence's
    key_lengths) are left as they were in these, and 0 in results made here."""
    f = _attn(q, k, v, offsets, key_offsets, key_lengths, causal, scale)
    shape = _shape(f, q, offsets, causal, cap, slopes, prefix)
    if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.device != q.device:
        raise ValueError("lse must be a contiguous float32 tensor of shape %s on %s" % (tuple(q.shape[:2]), q.device))
    lib = L.load()

    def call(handle):
        got = [torch.empty_like(like, memory_format=torch.contiguous_format) if t is None else t for t, like in ((dq, q), (dk, k), (dv, v))]
        at = [_heads_of(t, q, name, like.shape[0], like.shape[1]) for name, t, like in
              (("dout", dout, q), ("out", out, q), ("dq", got[0], q), ("dk", got[1], k), ("dv", got[2], v))]
        g = L.AttnGrads(at[0][0], at[1][0], lse.data_ptr(), *at[0][1:], *at[1][1:], at[2][0], at[3][0], at[4][0], *at[2][1:], *at[3][1:],
                        *at[4][1:])
        if dq is None or dk is None or dv is None:
            own = L.AttnGrads.from_buffer_copy(g)
            own.dq, own.dk, own.dv = [a[0] if t is None else None for a, t in zip(at[2:], (dq, dk, dv))]
            _check(lib.fuse_attention_zero_rest(f, own, handle))
        ws = _workspace(lib.fuse_attention_backward_bytes(f) if shape is None else lib.fuse_attention_shaped_backward_bytes(f, shape), q.device)
        if shape is None:
            _check(lib.fuse_attention_backward(f, g, ws.data_ptr(), ws.numel(), handle))
        else:
            _check(lib.fuse_attention_shaped_backward(f, shape, g, ws.data_ptr(), ws.numel(), handle))
        return tuple(got)

    return _run(q.device, stream, call)


# -------------------------------------------------------------------------- gradients ---

def _dense_cells(t, what):
    """A tensor whose cells lie side by side in memory, in whatever order of its dimensions."""
    _dtype(t, what)
    want = 1
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n > 1):
        if stride != want:
            raise ValueError("%s has gaps between its cells or overlaps itself" % what)
        want *= size
    return t


def _list(tensors, out):
    tensors = list(tensors)
    if not tensors:
        raise ValueError("no tensors")
    device = tensors[0].device
    if out is not None:
        out = list(out)
        if len(out) != len(tensors):
            raise ValueError("%d results for %d tensors" % (len(out), len(tensors)))
    index = device.index if device.type == "cuda" else -1
    cells = []                             # (data, out, count, dtype) of each, as L.Tensor has them
    for i, t in enumerate(tensors):
        flat, dtype, count = t.is_contiguous(), DTYPE.get(t.dtype), t.numel()
        if dtype is None or t.get_device() != index:
            _dtype(t, "tensor %d" % i)
            raise ValueError("tensor %d is on %s, not on %s" % (i, t.device, device))
        if not flat:
            _dense_cells(t, "tensor %d" % i)
        if out is None:
            cells += (t.data_ptr(), 0, count, dtype)
            continue
        o = out[i]
        if o.dtype is not t.dtype or o.get_device() != index:
            _like(o, t, "result %d" % i)
        if o.numel() != count or not (flat and o.is_contiguous() or o.shape == t.shape and o.stride() == t.stride()):
            raise ValueError("result %d is not laid out like its tensor" % i)
        cells += (t.data_ptr(), o.data_ptr(), count, dtype)
    return (ctypes.c_int64 * len(cells))(*cells), len(tensors), device


def _one_value(t, device, what):
    if t.dtype != torch.float64 or t.numel() != 1 or t.device != device:
        raise ValueError("%s must be one float64 value on %s" % (what, device))
    return t


def fuse_grad_norm(tensors, out=None, stream=None):
    """C: fuse_grad_norm.  The 2-norm over all cells of all tensors: one float64 value on the device."""
    arr, n, device = _list(tensors, None)
    if out is not None:
        _one_value(out, device, "out")
    lib = L.load()

    def call(handle):
        norm = torch.empty(1, dtype=torch.float64, device=device) if out is None else out
        ws = _workspace(lib.fuse_grad_norm_bytes(arr, n), device)
        _check(lib.fuse_grad_norm(arr, n, norm.data_ptr(), ws.data_ptr(), ws.numel(), handle))
        return norm

    return _run(device, stream, call)


def fuse_grad_clip(tensors, max_norm, eps=1e-6, norm=None, out=None, stream=None):
    """C: fuse_grad_clip.  Scales all tensors by min(1, max_norm / (norm + eps)), in place or into the tensors `out`; returns the
    norm (float64, on the device).  norm: None computes it; or one float64 value on the device that the program has already (such as the
    root of a sum over several processes)."""
    arr, n, device = _list(tensors, out)
    if norm is not None:
        _one_value(norm, device, "norm")
    lib = L.load()

    def call(handle):
        if norm is not None:
            _check(lib.fuse_grad_clip(arr, n, max_norm, eps, norm.data_ptr(), None, None, 0, handle))
            return norm
        found = torch.empty(1, dtype=torch.float64, device=device)
        ws = _workspace(lib.fuse_grad_norm_bytes(arr, n), device)
        _check(lib.fuse_grad_clip(arr, n, max_norm, eps, None, found.data_ptr(), ws.data_ptr(), ws.numel(), handle))
        return found

    return _run(device, stream, call)
