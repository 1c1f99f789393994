"""Operators of a transformer block: thin wrappers with the names of the C entry points (argument marshalling only).

Workspaces are torch tensors made on the call's stream, so a call that is captured into a HIP graph keeps its own in the
graph's memory pool, and two graphs or streams share none.
"""
import ctypes
from collections import namedtuple
from contextlib import contextmanager

import torch

from . import _lib as L
from .api import SIDE, _check

NORM = {"rms": 0, "layer": 1}
DTYPE = {torch.float64: 0, torch.float32: 1, torch.bfloat16: 2, torch.float16: 3}

BlockGrads = namedtuple("BlockGrads", "dx dz dgate dpost dpost_bias dpre dpre_bias")
"""Gradients of fuse_block_norm; None where the call had no such input."""


@contextmanager
def _on(device, stream):
    """The device, and the stream on it (default: its current one), that a call runs on; yields the stream's handle.
    Allocations inside belong to that stream."""
    if device.type != "cuda":
        raise ValueError("tensors must be CUDA (HIP) tensors, got device %s" % device)
    if stream is not None and not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    if stream is not None and stream.device != device:
        raise ValueError("the stream is on %s, the tensors are on %s" % (stream.device, device))
    if stream is None and device.index == torch.cuda.current_device():
        yield ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)
        return
    with torch.cuda.device(device):
        if stream is None:
            stream = torch.cuda.current_stream(device)
        with torch.cuda.stream(stream):
            yield ctypes.c_void_p(stream.cuda_stream)


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def _like(t, x, what):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % what)
    if t.device != x.device:
        raise ValueError("%s is on %s, not on %s" % (what, t.device, x.device))
    if t.dtype != x.dtype:
        raise TypeError("%s is %s, not %s" % (what, t.dtype, x.dtype))
    return t


def _dtype(x, what):
    if not isinstance(x, torch.Tensor) or x.dtype not in DTYPE:
        raise TypeError("%s must be a float64, float32, bfloat16 or float16 tensor" % what)
    return DTYPE[x.dtype]


# ------------------------------------------------------------------------------ norms ---

def _rows_of(t, x, what):
    """Pointer and leading dimension of a matrix of x's shape with unit column stride."""
    _like(t, x, what)
    if t.shape != x.shape:
        raise ValueError("%s has shape %s, not %s" % (what, tuple(t.shape), tuple(x.shape)))
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("%s needs unit column stride" % what)
    return t.data_ptr(), t.stride(0) if rows > 1 else cols


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
    b = L.Block(dtype=dtype, norm=NORM[kind], rows=rows, cols=cols, eps=float(eps), scale=float(scale), gate_kind=-1)
    if z is not None:
        b.z, b.z_ld = _rows_of(z, x, "z")
    for name, p in (("post", post), ("pre", pre)):
        w, bias = _weights(p)
        if w is not None:
            setattr(b, name + "_weight", _vector(w, x, cols, name + " weight"))
        if bias is not None:
            setattr(b, name + "_bias", _vector(bias, x, cols, name + " bias"))
    gk, gt = (None, None) if gate is None else gate
    if gk is not None:
        if gk not in ("rowvec", "colvec", "matrix"):
            raise ValueError("a gate is ('rowvec' | 'colvec' | 'matrix', tensor), not %r" % (gk,))
        b.gate_kind = SIDE[gk]
        if gk == "rowvec":
            b.gate = _vector(gt, x, cols, "gate")
        elif gk == "matrix":
            b.gate, b.gate_ld = _rows_of(gt, x, "gate")
        else:
            _like(gt, x, "gate")
            if gt.dim() != 1 or gt.numel() != rows:
                raise ValueError("gate must be a vector of %d values" % rows)
            b.gate, b.gate_ld = gt.data_ptr(), gt.stride(0) if rows > 1 else 1
        if not gt.numel():
            b.gate = x.data_ptr() or 16      # (no rows: never read)
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
    with _on(x.device, stream) as handle:
        if z is not None and h is None:
            h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if pre is not None and y is None:
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        hp, h_ld = _rows_of(h, x, "h") if h is not None else (None, 0)
        yp, y_ld = _rows_of(y, x, "y") if y is not None else (None, 0)
        if x.numel():
            _check(L.load().fuse_block_norm(ctypes.byref(b), xp, x_ld, hp, h_ld, yp, y_ld, handle))
    return (x if h is None else h), y


def fuse_block_norm_backward(dh, dy, h, z=None, gate=None, scale=1.0, post=None, pre=None, kind="rms", eps=1e-6, stream=None):
    """C: fuse_block_norm_backward.  Gradients of fuse_block_norm from those of its results (one of them may be None: zero),
    its h (x where there was no z) and its other inputs: a BlockGrads."""
    like = h if h is not None else dh
    b, gk, gt = _block(like, z, gate, scale, post, pre, kind, eps, "h")
    (post_w, post_b), (pre_w, pre_b) = _weights(post), _weights(pre)
    lib = L.load()
    with _on(like.device, stream) as handle:
        def new(t):
            return None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device)

        got = BlockGrads(new(like), new(z), new(gt), new(post_w), new(post_b), new(pre_w), new(pre_b))
        if like.numel() == 0:
            for t in got:
                if t is not None:
                    t.zero_()
            return got
        g = L.BlockGrads(dx=got.dx.data_ptr(), dx_ld=like.shape[1], dgate_ld=like.shape[1] if gk == "matrix" else 1)
        if z is not None:
            g.dz, g.dz_ld = got.dz.data_ptr(), like.shape[1]
        for name, t in (("dgate", got.dgate), ("dpost_weight", got.dpost), ("dpost_bias", got.dpost_bias),
                        ("dpre_weight", got.dpre), ("dpre_bias", got.dpre_bias)):
            if t is not None:
                setattr(g, name, t.data_ptr())
        nbytes = lib.fuse_block_norm_backward_bytes(ctypes.byref(b))
        ws = _workspace(nbytes, like.device)
        args = []
        for t, what in ((dh, "dh"), (dy, "dy"), (h, "h")):
            args += _rows_of(t, like, what) if t is not None else (None, 0)
        _check(lib.fuse_block_norm_backward(ctypes.byref(b), *args, ctypes.byref(g), ws.data_ptr(), ws.numel(), handle))
    return got


# -------------------------------------------------------------------------- attention ---

def _heads_of(t, like, what, tokens=None, heads=None):
    """(pointer, stride between tokens, stride between heads) of a (tokens, heads, dim) tensor with unit stride along dim."""
    _like(t, like, what)
    if t.dim() != 3 or t.shape[2] != like.shape[2]:
        raise ValueError("%s must be (tokens, heads, %d)" % (what, like.shape[2]))
    if (tokens is not None and t.shape[0] != tokens) or (heads is not None and t.shape[1] != heads):
        raise ValueError("%s has shape %s, not (%s, %s, %d)" % (what, tuple(t.shape), tokens, heads, like.shape[2]))
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError("%s needs unit stride along dim" % what)
    dim = t.shape[2]
    return (t.data_ptr(), t.stride(0) if t.shape[0] > 1 else dim * max(t.shape[1], 1), t.stride(1) if t.shape[1] > 1 else dim)


def _attn(q, k, v, offsets, key_offsets, key_lengths, causal, scale):
    dtype = _dtype(q, "q")
    if q.dim() != 3 or k.dim() != 3 or q.shape[1] < 1 or k.shape[1] < 1 or q.shape[2] < 1:
        raise ValueError("q, k and v must be (tokens, heads, dim)")
    f = L.Attn(dtype=dtype, heads=q.shape[1], kv_heads=k.shape[1], dim=q.shape[2], causal=int(bool(causal)),
               q_tokens=q.shape[0], k_tokens=k.shape[0], scale=float(scale) if scale is not None else q.shape[2] ** -0.5)
    f.q, f.q_token_ld, f.q_head_ld = _heads_of(q, q, "q")
    f.k, f.k_token_ld, f.k_head_ld = _heads_of(k, q, "k")
    f.v, f.v_token_ld, f.v_head_ld = _heads_of(v, q, "v", k.shape[0], k.shape[1])
    if offsets is None or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets must be a vector of the number of sequences + 1 values")
    f.seqs = offsets.numel() - 1
    if key_lengths is not None and key_offsets is None:
        raise ValueError("key_lengths needs key_offsets")
    for t, what, count in ((offsets, "offsets", f.seqs + 1), (key_offsets, "key_offsets", f.seqs + 1), (key_lengths, "key_lengths", f.seqs)):
        if t is None:
            continue
        if t.dtype not in (torch.int32, torch.int64) or t.dtype != offsets.dtype:
            raise TypeError("%s must be int32 or int64, like offsets" % what)
        if t.device != q.device:
            raise ValueError("%s is on %s, not on %s" % (what, t.device, q.device))
        if t.dim() != 1 or t.numel() != count or not t.is_contiguous():
            raise ValueError("%s must be a contiguous vector of %d values" % (what, count))
    f.offsets_are_64 = int(offsets.dtype == torch.int64)
    f.q_offsets = offsets.data_ptr()
    f.k_offsets = key_offsets.data_ptr() if key_offsets is not None else None
    f.k_lengths = key_lengths.data_ptr() if key_lengths is not None else None
    return f


def fuse_attention(q, k, v, offsets, key_offsets=None, key_lengths=None, causal=True, scale=None, out=None, lse=None, stream=None):
    """C: fuse_attention.  softmax(scale * q k^T + mask) v for packed sequences; returns (out, lse).

    q: (tokens, heads, dim), k and v: (key tokens, key heads, dim), bfloat16 or float16, heads a multiple of key heads; parts of
    one projection can be passed as they are.  offsets: the sequences' first queries and the end of the last one; key_offsets likewise
    for the keys (None: the same), with key_lengths only so many keys from each sequence's first one on (a cache with room).
    causal: the last query sees all keys, the one before it all but the last, and so on.  scale: None is 1 / sqrt(dim).  lse:
    (tokens, heads) float32.  Rows that belong to no sequence are not written: in results made here they hold anything."""
    f = _attn(q, k, v, offsets, key_offsets, key_lengths, causal, scale)
    lib = L.load()
    with _on(q.device, stream) as handle:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        elif lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.device != q.device:
            raise ValueError("lse must be a contiguous float32 tensor of shape %s on %s" % (tuple(q.shape[:2]), q.device))
        op, o_token, o_head = _heads_of(out, q, "out", q.shape[0], q.shape[1])
        nbytes = lib.fuse_attention_bytes(ctypes.byref(f))
        ws = _workspace(nbytes, q.device) if nbytes else None
        _check(lib.fuse_attention(ctypes.byref(f), op, o_token, o_head, lse.data_ptr(), ws.data_ptr() if nbytes else None, nbytes, handle))
    return out, lse


def fuse_attention_backward(dout, q, k, v, out, lse, offsets, key_offsets=None, key_lengths=None, causal=True, scale=None,
                            dq=None, dk=None, dv=None, stream=None):
    """C: fuse_attention_backward.  Gradients (dq, dk, dv) of fuse_attention's out, given its results and its other arguments."""
    f = _attn(q, k, v, offsets, key_offsets, key_lengths, causal, scale)
    if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.device != q.device:
        raise ValueError("lse must be a contiguous float32 tensor of shape %s on %s" % (tuple(q.shape[:2]), q.device))
    lib = L.load()
    with _on(q.device, stream) as handle:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
        g = L.AttnGrads(lse=lse.data_ptr())
        for name, t, like in (("dout", dout, q), ("out", out, q), ("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
            p, token, head = _heads_of(t, q, name, like.shape[0], like.shape[1])
            setattr(g, name, p)
            setattr(g, name + "_token_ld", token)
            setattr(g, name + "_head_ld", head)
        nbytes = lib.fuse_attention_backward_bytes(ctypes.byref(f))
        ws = _workspace(nbytes, q.device)
        _check(lib.fuse_attention_backward(ctypes.byref(f), ctypes.byref(g), ws.data_ptr(), ws.numel(), handle))
    return dq, dk, dv


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
    arr = (L.Tensor * len(tensors))()
    for i, t in enumerate(tensors):
        if not t.is_contiguous():
            _dense_cells(t, "tensor %d" % i)
        dtype = DTYPE.get(t.dtype)
        if dtype is None or t.device != device:
            _dtype(t, "tensor %d" % i)
            raise ValueError("tensor %d is on %s, not on %s" % (i, t.device, device))
        a = arr[i]
        a.data, a.count, a.dtype = t.data_ptr(), t.numel(), dtype
        if out is not None:
            o = out[i]
            _like(o, t, "result %d" % i)
            if o.shape != t.shape or (o.stride() != t.stride() and not (o.is_contiguous() and t.is_contiguous())):
                raise ValueError("result %d is not laid out like its tensor" % i)
            a.out = o.data_ptr()
    return arr, device


def fuse_grad_norm(tensors, out=None, stream=None):
    """C: fuse_grad_norm.  The 2-norm over all cells of all tensors: one float64 value on the device."""
    arr, device = _list(tensors, None)
    lib = L.load()
    with _on(device, stream) as handle:
        if out is None:
            out = torch.empty(1, dtype=torch.float64, device=device)
        elif out.dtype != torch.float64 or out.numel() != 1 or out.device != device:
            raise ValueError("out must be one float64 value on %s" % device)
        ws = _workspace(lib.fuse_grad_norm_bytes(arr, len(arr)), device)
        _check(lib.fuse_grad_norm(arr, len(arr), out.data_ptr(), ws.data_ptr(), ws.numel(), handle))
    return out


def fuse_grad_clip(tensors, max_norm, eps=1e-6, norm=None, out=None, stream=None):
    """C: fuse_grad_clip.  Scales all tensors by min(1, max_norm / (norm + eps)), in place or into the tensors `out`; returns the
    norm (float64, on the device).  norm: None computes it; or one float64 value on the device that the program has already (such as the
    root of a sum over several processes)."""
    arr, device = _list(tensors, out)
    lib = L.load()
    with _on(device, stream) as handle:
        if norm is not None:
            if norm.dtype != torch.float64 or norm.numel() != 1 or norm.device != device:
                raise ValueError("norm must be one float64 value on %s" % device)
            _check(lib.fuse_grad_clip(arr, len(arr), float(max_norm), float(eps), norm.data_ptr(), None, None, 0, handle))
            return norm
        norm = torch.empty(1, dtype=torch.float64, device=device)
        ws = _workspace(lib.fuse_grad_norm_bytes(arr, len(arr)), device)
        _check(lib.fuse_grad_clip(arr, len(arr), float(max_norm), float(eps), None, norm.data_ptr(), ws.data_ptr(), ws.numel(), handle))
    return norm
