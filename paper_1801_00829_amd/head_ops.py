"""Operators on the heads of a projection: thin wrappers with the names of the C entry points (argument marshalling only)."""
import struct
from collections import namedtuple

import torch

from . import _lib as L
from .api import _check
from .block_ops import DTYPE, _cap, _dtype, _heads_of, _places, _row, _run, _vector, _workspace

PAIRS = {"halves": 0, "neighbours": 1}

RotaryGrads = namedtuple("RotaryGrads", "dq dk dq_weight dk_weight")
"""Gradients of fuse_qk_rotary; None where the call had no such input."""

Cache = namedtuple("Cache", "k v k_scale v_scale")
"""A cache of keys and values in 8 bits: k, v (pages, key heads, places per page, dim) float8_e4m3fn, with equal strides; k_scale, v_scale
(pages, key heads, places per page) float32, likewise."""


# ------------------------------------------------------------- norms and rotary positions ---

# (descriptors are packed in one go: filling a ctypes structure takes several times as long, and small calls are bound by that)
_ROTARY = struct.Struct("@iiiiiiiiiii4x qqPPPPd PPqqqq".replace(" ", ""))
_ROTARY_GRADS = struct.Struct("@PPqqqqPPqqqqPP")


def _weight(t, like, dim, what):
    if t is None:
        return 0
    if t.dtype is like.dtype and t.get_device() == like.get_device() and t.shape == (dim,) and (t.stride(0) == 1 or dim == 1):
        return t.data_ptr()
    return _vector(t, like, dim, what)


def _rotary(q, k, positions, freqs, q_weight, k_weight, sections, pairs, eps, what):
    """Packs the descriptor of a call on tensors of these shapes, once it is given q's and k's places (pointer, strides)."""
    dtype = DTYPE.get(q.dtype) if isinstance(q, torch.Tensor) else None
    if dtype is None:
        _dtype(q, what)
    shape = q.shape
    if len(shape) != 3 or shape[1] < 1 or shape[2] < 1:
        raise ValueError("%s must be (tokens, heads, dim)" % what)
    tokens, heads, dim = shape
    kind = PAIRS.get(pairs)
    if kind is None:
        raise ValueError("pairs is 'halves' or 'neighbours', not %r" % (pairs,))
    kv_heads = 0
    if k is not None:
        if k.dim() != 3 or k.shape[1] < 1:
            raise ValueError("keys must be (tokens, heads, dim); without any, pass None")
        kv_heads = k.shape[1]
    elif k_weight is not None:
        raise ValueError("k_weight needs keys")
    if not isinstance(positions, torch.Tensor) or (positions.dtype is not torch.int32 and positions.dtype is not torch.int64):
        raise TypeError("positions must be an int32 or int64 tensor")
    if not isinstance(freqs, torch.Tensor) or freqs.dtype is not torch.float64:
        raise TypeError("freqs must be a float64 tensor")
    if not positions.get_device() == freqs.get_device() == q.get_device():
        raise ValueError("positions are on %s and freqs on %s, not on %s" % (positions.device, freqs.device, q.device))
    if freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError("freqs must be a contiguous vector of a value per pair")
    half, at = freqs.numel(), positions.shape
    if sections is None:
        sections, axes = (half, 0, 0, 0), 1
    else:
        axes = len(sections)
        if not 1 <= axes <= 4:
            raise ValueError("sections has a number of pairs for each of 1 to 4 axes")
        if sum(sections) != half:
            raise ValueError("sections have %d pairs, freqs has %d" % (sum(sections), half))
        sections = tuple(sections) + (0,) * (4 - axes)
    if len(at) == 1 and axes == 1:
        ld, fits, step = tokens, at[0] == tokens, positions.stride(0)
    else:
        fits = len(at) == 2 and at[0] == axes and at[1] == tokens
        ld, step = positions.stride() if fits else (0, 1)
    if not fits:
        raise ValueError("positions must be (%s%d), not %s" % ("" if axes == 1 else "%d, " % axes, tokens, tuple(at)))
    if step != 1 and tokens > 1:
        raise ValueError("positions needs unit stride along the tokens")
    qw, kw = _weight(q_weight, q, dim, "q_weight"), _weight(k_weight, q, dim, "k_weight")
    return lambda at_q, at_k: _ROTARY.pack(dtype, heads, kv_heads, dim, kind, axes, positions.dtype is torch.int64, *sections, tokens, ld,
                                           positions.data_ptr(), freqs.data_ptr(), qw, kw, eps, at_q[0], at_k[0], *at_q[1:], *at_k[1:])


_NONE = (0, 0, 0)


def _at(t, like, what, tokens, heads):
    """_heads_of, in short where a tensor is as it should be."""
    if isinstance(t, torch.Tensor) and t.dtype is like.dtype and t.get_device() == like.get_device():
        shape, (token, head, step) = t.shape, t.stride() if t.dim() == 3 else (0, 0, 0)
        if step == 1 and shape[0] == tokens > 1 and shape[1] == heads > 1 and shape[2] == like.shape[2]:
            return t.data_ptr(), token, head
    return _heads_of(t, like, what, tokens, heads)


def _result(t, like, what):
    """A result of like's shape to write to, and its place."""
    if t is None:
        _, heads, dim = like.shape
        t = torch.empty_like(like, memory_format=torch.contiguous_format)
        return t, (t.data_ptr(), heads * dim, dim)
    return t, _at(t, like, what, *like.shape[:2])


def _pointer(t):
    return 0 if t is None else t.data_ptr()


def fuse_qk_rotary(q, k, positions, freqs, q_weight=None, k_weight=None, sections=None, pairs="halves", eps=1e-6, q_out=None, k_out=None,
                   stream=None):
    """C: fuse_qk_rotary.  Norms of the heads (where there is a weight) and their rotation by positions; returns (q_out, k_out).

    q: (tokens, heads, dim), k: (tokens, key heads, dim) or None; parts of one projection can be passed as they are.  freqs: float64, radians
    per position of every pair of dims that turns.  positions: (tokens,), or with sections (pairs of axis 0, of axis 1, ...) a row for
    every axis.  pairs: "halves" (dims i and i + number of pairs) or "neighbours" (2 i and 2 i + 1).  q_out, k_out: tensors to write to; they
    may be q and k themselves."""
    pack = _rotary(q, k, positions, freqs, q_weight, k_weight, sections, pairs, eps, "q")
    tokens, heads, _ = q.shape
    f = pack(_at(q, q, "q", tokens, heads), _NONE if k is None else _at(k, q, "k", tokens, k.shape[1]))
    if k is None and k_out is not None:
        raise ValueError("k_out needs keys")

    def call(handle):
        got_q, at_q = _result(q_out, q, "q_out")
        got_k, at_k = (None, _NONE) if k is None else _result(k_out, k, "k_out")
        _check(L.load().fuse_qk_rotary(f, *at_q, *at_k, handle))
        return got_q, got_k

    return _run(q.device, stream, call)


def fuse_qk_rotary_backward(dq_out, dk_out, q, k, positions, freqs, q_weight=None, k_weight=None, sections=None, pairs="halves", eps=1e-6,
                            dq=None, dk=None, stream=None):
    """C: fuse_qk_rotary_backward.  Gradients of fuse_qk_rotary from those of its results and its other arguments: a RotaryGrads.

    q and k are only read where there is a norm, and may be None without one.  dq, dk: tensors to write to; they may be dq_out and dk_out, or
    q and k, themselves."""
    pack = _rotary(dq_out, dk_out, positions, freqs, q_weight, k_weight, sections, pairs, eps, "dq_out")
    if dk_out is None and dk is not None:
        raise ValueError("dk needs keys")
    tokens, heads, _ = dq_out.shape
    at_dq = _at(dq_out, dq_out, "dq_out", tokens, heads)
    at_dk = _NONE if dk_out is None else _at(dk_out, dq_out, "dk_out", tokens, dk_out.shape[1])
    f = pack(_NONE if q_weight is None else _at(q, dq_out, "q", tokens, heads),
             _NONE if k_weight is None else _at(k, dq_out, "k", tokens, dk_out.shape[1]))
    lib = L.load()

    def call(handle):
        got_q, to_q = _result(dq, dq_out, "dq")
        got_k, to_k = (None, _NONE) if dk_out is None else _result(dk, dk_out, "dk")
        got_qw, got_kw = [None if w is None else torch.empty_like(w) for w in (q_weight, k_weight)]
        g = _ROTARY_GRADS.pack(at_dq[0], at_dk[0], *at_dq[1:], *at_dk[1:], to_q[0], to_k[0], *to_q[1:], *to_k[1:], _pointer(got_qw),
                               _pointer(got_kw))
        nbytes = lib.fuse_qk_rotary_backward_bytes(f)
        ws = _workspace(nbytes, dq_out.device) if nbytes else None
        _check(lib.fuse_qk_rotary_backward(f, g, _pointer(ws), nbytes, handle))
        return RotaryGrads(got_q, got_k, got_qw, got_kw)

    return _run(dq_out.device, stream, call)


# ------------------------------------------------------------------------ cache in 8 bits ---

def cache_new(pages, page_size, kv_heads, dim, device="cuda"):
    """A Cache of zeros."""
    data = [torch.zeros((pages, kv_heads, page_size, dim), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)]
    return Cache(*data, *[torch.zeros((pages, kv_heads, page_size), dtype=torch.float32, device=device) for _ in range(2)])


_CACHE = struct.Struct("@iiiiqqqqPPPPqqqqqPqqPP")
_CACHE_QUERY = struct.Struct("@PqqiiddPP")


def _cache(cache, x, offsets, page_table, lengths):
    """(packed descriptor, key heads) of a call with packed arrays (tokens, any, dim) like x."""
    dtype = DTYPE.get(x.dtype) if isinstance(x, torch.Tensor) else None
    if dtype is None:
        _dtype(x, "packed rows")
    k, v, k_scale, v_scale = cache
    index, shape, strides = x.get_device(), k.shape, k.stride()
    if not (k.dtype is v.dtype is torch.float8_e4m3fn and k_scale.dtype is v_scale.dtype is torch.float32 and
            k.get_device() == v.get_device() == k_scale.get_device() == v_scale.get_device() == index):
        for t, name, want in ((k, "k", torch.float8_e4m3fn), (v, "v", torch.float8_e4m3fn), (k_scale, "k_scale", torch.float32),
                              (v_scale, "v_scale", torch.float32)):
            if t.dtype is not want:
                raise TypeError("the cache's %s must be a %s tensor" % (name, want))
            if t.get_device() != index:
                raise ValueError("the cache's %s is on %s, not on %s" % (name, t.device, x.device))
    if len(shape) != 4 or v.shape != shape or k_scale.shape != shape[:3] or v_scale.shape != shape[:3]:
        raise ValueError("the cache's k and v must be (pages, key heads, places per page, dim), their scales the same without dim")
    scales = k_scale.stride()
    pages, kv_heads, page_size, dim = shape
    if dim != x.shape[2] or kv_heads < 1 or page_size < 1:
        raise ValueError("the cache has shape %s, rows have dim %d" % (tuple(shape), x.shape[2]))
    if (v.stride() != strides or v_scale.stride() != scales) and pages:
        raise ValueError("the cache's k and v, and their scales, must have equal strides")
    if (strides[3] != 1 and dim > 1) or (scales[2] != 1 and page_size > 1):
        raise ValueError("the cache needs unit stride along dim, and its scales along the places")
    if offsets is None or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets must be a vector of the number of sequences + 1 values")
    kind, seqs = offsets.dtype, offsets.numel() - 1
    if kind is not torch.int32 and kind is not torch.int64:
        raise TypeError("offsets must be int32 or int64")
    if not (lengths.dtype is kind and offsets.get_device() == lengths.get_device() == index and lengths.dim() == 1 and lengths.numel() == seqs and
            offsets.is_contiguous() and lengths.is_contiguous()):
        _places(offsets, offsets, x.device, seqs + 1, "offsets")
        _places(lengths, offsets, x.device, seqs, "lengths")
    if page_table.dtype is not torch.int32:
        raise TypeError("page_table must be an int32 tensor")
    if page_table.get_device() != index:
        raise ValueError("page_table is on %s, not on %s" % (page_table.device, x.device))
    table, steps = page_table.shape, page_table.stride()
    if len(table) != 2 or table[0] != seqs or (table[1] > 1 and steps[1] != 1):
        raise ValueError("page_table must be (%d, pages of a sequence) with unit stride along the pages" % seqs)
    # (a stride of a single page, head or place means nothing)
    return _CACHE.pack(dtype, kv_heads, dim, kind is torch.int64, x.shape[0], seqs, pages, page_size, k.data_ptr(), v.data_ptr(),
                       k_scale.data_ptr(), v_scale.data_ptr(), strides[0] if pages > 1 else 0, strides[1] if kv_heads > 1 else 0,
                       strides[2] if page_size > 1 else 0, scales[0] if pages > 1 else 0, scales[1] if kv_heads > 1 else 0,
                       page_table.data_ptr(), steps[0] if seqs > 1 else table[1], table[1], offsets.data_ptr(), lengths.data_ptr()), kv_heads


def fuse_cache_write(k, v, cache, offsets, page_table, lengths, stream=None):
    """C: fuse_cache_write.  Writes the keys and values of new tokens, rounded to 8 bits with a scale per token and head, into a Cache.

    k, v: (tokens, key heads, dim), bfloat16 or float16; parts of one projection can be passed as they are.  offsets: the sequences' first new tokens
    and the end of the last one; lengths: their keys, the new ones among them (the last ones): a new token goes to the place of its key.
    page_table: (sequences, pages) int32, the pages of every sequence in order; tokens that it has no place for are not written."""
    if k.dim() != 3:
        raise ValueError("k must be (tokens, heads, dim)")
    f, kv_heads = _cache(cache, k, offsets, page_table, lengths)
    at_k, at_v = _at(k, k, "k", k.shape[0], kv_heads), _at(v, k, "v", k.shape[0], kv_heads)
    return _run(k.device, stream, lambda handle: _check(L.load().fuse_cache_write(f, *at_k, *at_v, handle)))


def fuse_attention_cache(q, cache, offsets, page_table, lengths, causal=True, scale=None, cap=None, slopes=None, tree=None, out=None, lse=None,
                         stream=None):
    """C: fuse_attention_cache.  Attention of new tokens over a Cache that holds their keys and values already; returns (out, lse).

    q: (tokens, heads, dim), bfloat16 or float16, heads a multiple of the cache's.  offsets, page_table, lengths: as in fuse_cache_write.  causal:
    the last query sees all keys, the one before it all but the last, and so on.  scale: None is 1 / sqrt(dim).  cap: scores become
    cap * tanh(score / cap).  slopes: (heads,) float32, slopes[h] * |distance| is taken off the scores.  tree: (tokens,) int64, of the new tokens of
    its sequence a query sees those whose bits are set in its word (up to 64; its own has to be set too).  lse: (tokens, heads) float32.  Rows that
    belong to no sequence are not written: in results made here they hold anything."""
    if q.dim() != 3 or q.shape[1] < 1:
        raise ValueError("q must be (tokens, heads, dim)")
    f, _ = _cache(cache, q, offsets, page_table, lengths)
    n, heads, dim = q.shape
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (n, heads) or not lse.is_contiguous() or lse.device != q.device):
        raise ValueError("lse must be a contiguous float32 tensor of shape %s on %s" % ((n, heads), q.device))
    d = _CACHE_QUERY.pack(*_at(q, q, "q", n, heads), heads, 1 if causal else 0, dim ** -0.5 if scale is None else scale, _cap(cap),
                          0 if slopes is None else _row(slopes, q, torch.float32, heads, "slopes"),
                          0 if tree is None else _row(tree, q, torch.int64, n, "tree"))
    lib = L.load()

    def call(handle):
        l = torch.empty((n, heads), dtype=torch.float32, device=q.device) if lse is None else lse
        o, at = _result(out, q, "out")
        nbytes = lib.fuse_attention_cache_bytes(f, d)
        ws = _workspace(nbytes, q.device) if nbytes else None
        _check(lib.fuse_attention_cache(f, d, *at, l.data_ptr(), _pointer(ws), nbytes, handle))
        return o, l

    return _run(q.device, stream, call)
