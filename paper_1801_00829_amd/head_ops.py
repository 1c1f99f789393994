"""Operators on the heads of a projection: thin wrappers with the names of the C entry points (argument marshalling only)."""
from collections import namedtuple

import torch

from . import _lib as L
from .api import _check
from .block_ops import _cap, _dtype, _heads_of, _like, _places, _row, _run, _vector, _workspace

PAIRS = {"halves": 0, "neighbours": 1}

RotaryGrads = namedtuple("RotaryGrads", "dq dk dq_weight dk_weight")
"""Gradients of fuse_qk_rotary; None where the call had no such input."""

Cache = namedtuple("Cache", "k v k_scale v_scale")
"""A cache of keys and values in 8 bits: k, v (pages, key heads, places per page, dim) float8_e4m3fn, with equal strides; k_scale, v_scale
(pages, key heads, places per page) float32, likewise."""


# ------------------------------------------------------------- norms and rotary positions ---

def _rotary(q, k, positions, freqs, q_weight, k_weight, sections, pairs, eps, what):
    """Descriptor of a call on tensors of these shapes; q and k themselves, with their strides, are put in by the caller."""
    dtype = _dtype(q, what)
    if q.dim() != 3 or q.shape[1] < 1 or q.shape[2] < 1:
        raise ValueError("%s must be (tokens, heads, dim)" % what)
    if pairs not in PAIRS:
        raise ValueError("pairs is 'halves' or 'neighbours', not %r" % (pairs,))
    tokens, heads, dim = q.shape
    if k is not None and k.shape[1] < 1:
        raise ValueError("keys have no heads: pass None")
    if k is None and k_weight is not None:
        raise ValueError("k_weight needs keys")
    if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.int64):
        raise TypeError("positions must be an int32 or int64 tensor")
    if not isinstance(freqs, torch.Tensor) or freqs.dtype is not torch.float64:
        raise TypeError("freqs must be a float64 tensor")
    for t, name in ((positions, "positions"), (freqs, "freqs")):
        if t.device != q.device:
            raise ValueError("%s is on %s, not on %s" % (name, t.device, q.device))
    if freqs.dim() != 1 or (freqs.numel() > 1 and freqs.stride(0) != 1):
        raise ValueError("freqs must be a contiguous vector of a value per pair")
    if sections is None:
        sections = (freqs.numel(),)
    if not 1 <= len(sections) <= 4:
        raise ValueError("sections has a number of pairs for each of 1 to 4 axes")
    if sum(sections) != freqs.numel():
        raise ValueError("sections have %d pairs, freqs has %d" % (sum(sections), freqs.numel()))
    axes = len(sections)
    if positions.shape != ((axes, tokens) if positions.dim() == 2 else (tokens,)) or (positions.dim() == 1 and axes > 1):
        raise ValueError("positions must be (%s%d), not %s" % ("" if axes == 1 else "%d, " % axes, tokens, tuple(positions.shape)))
    if tokens > 1 and positions.stride(-1) != 1:
        raise ValueError("positions needs unit stride along the tokens")
    ld = positions.stride(0) if positions.dim() == 2 and axes > 1 else tokens
    return L.Rotary(dtype, heads, 0 if k is None else k.shape[1], dim, PAIRS[pairs], axes, 1 if positions.dtype is torch.int64 else 0,
                    tuple(sections), tokens, ld, positions.data_ptr(), freqs.data_ptr(),
                    None if q_weight is None else _vector(q_weight, q, dim, "q_weight"),
                    None if k_weight is None else _vector(k_weight, q, dim, "k_weight"), eps)


def _new(t):
    return None if t is None else torch.empty_like(t, memory_format=torch.contiguous_format)


def fuse_qk_rotary(q, k, positions, freqs, q_weight=None, k_weight=None, sections=None, pairs="halves", eps=1e-6, q_out=None, k_out=None,
                   stream=None):
    """C: fuse_qk_rotary.  Norms of the heads (where there is a weight) and their rotation by positions; returns (q_out, k_out).

    q: (tokens, heads, dim), k: (tokens, key heads, dim) or None; parts of one projection can be passed as they are.  freqs: float64, radians
    per position of every pair of dims that turns.  positions: (tokens,), or with sections (pairs of axis 0, of axis 1, ...) a row for
    every axis.  pairs: "halves" (dims i and i + number of pairs) or "neighbours" (2 i and 2 i + 1).  q_out, k_out: tensors to write to; they
    may be q and k themselves."""
    f = _rotary(q, k, positions, freqs, q_weight, k_weight, sections, pairs, eps, "q")
    f.q, f.q_token_ld, f.q_head_ld = _heads_of(q, q, "q")
    if k is not None:
        f.k, f.k_token_ld, f.k_head_ld = _heads_of(k, q, "k", q.shape[0])
    elif k_out is not None:
        raise ValueError("k_out needs keys")

    def call(handle):
        got_q, got_k = _new(q) if q_out is None else q_out, _new(k) if k_out is None else k_out
        at_q = _heads_of(got_q, q, "q_out", q.shape[0], q.shape[1])
        at_k = (None, 0, 0) if k is None else _heads_of(got_k, q, "k_out", k.shape[0], k.shape[1])
        _check(L.load().fuse_qk_rotary(f, *at_q, *at_k, handle))
        return got_q, got_k

    return _run(q.device, stream, call)


def fuse_qk_rotary_backward(dq_out, dk_out, q, k, positions, freqs, q_weight=None, k_weight=None, sections=None, pairs="halves", eps=1e-6,
                            dq=None, dk=None, stream=None):
    """C: fuse_qk_rotary_backward.  Gradients of fuse_qk_rotary from those of its results and its other arguments: a RotaryGrads.

    q and k are only read where there is a norm, and may be None without one.  dq, dk: tensors to write to; they may be dq_out and dk_out, or
    q and k, themselves."""
    f = _rotary(dq_out, dk_out, positions, freqs, q_weight, k_weight, sections, pairs, eps, "dq_out")
    if dk_out is None and dk is not None:
        raise ValueError("dk needs keys")
    at = [_heads_of(dq_out, dq_out, "dq_out"), (None, 0, 0) if dk_out is None else _heads_of(dk_out, dq_out, "dk_out", dq_out.shape[0])]
    if q_weight is not None:
        f.q, f.q_token_ld, f.q_head_ld = _heads_of(_like(q, dq_out, "q"), dq_out, "q", *dq_out.shape[:2])
    if k_weight is not None:
        f.k, f.k_token_ld, f.k_head_ld = _heads_of(_like(k, dq_out, "k"), dq_out, "k", *dk_out.shape[:2])
    lib = L.load()

    def call(handle):
        got = RotaryGrads(_new(dq_out) if dq is None else dq, _new(dk_out) if dk is None else dk, _new(q_weight), _new(k_weight))
        at_q = _heads_of(got.dq, dq_out, "dq", *dq_out.shape[:2])
        at_k = (None, 0, 0) if dk_out is None else _heads_of(got.dk, dq_out, "dk", *dk_out.shape[:2])
        g = L.RotaryGrads(at[0][0], at[1][0], *at[0][1:], *at[1][1:], at_q[0], at_k[0], *at_q[1:], *at_k[1:],
                          *[None if t is None else t.data_ptr() for t in got[2:]])
        nbytes = lib.fuse_qk_rotary_backward_bytes(f)
        ws = _workspace(nbytes, dq_out.device) if nbytes else None
        _check(lib.fuse_qk_rotary_backward(f, g, ws.data_ptr() if nbytes else None, nbytes, handle))
        return got

    return _run(dq_out.device, stream, call)


# ------------------------------------------------------------------------ cache in 8 bits ---

def cache_new(pages, page_size, kv_heads, dim, device="cuda"):
    """A Cache of zeros."""
    data = [torch.zeros((pages, kv_heads, page_size, dim), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)]
    return Cache(*data, *[torch.zeros((pages, kv_heads, page_size), dtype=torch.float32, device=device) for _ in range(2)])


def _cache(cache, x, tokens, offsets, page_table, lengths):
    """Descriptor of a call with packed arrays like x."""
    dtype = _dtype(x, "packed rows")
    k, v, k_scale, v_scale = cache
    for t, name, want in ((k, "k", torch.float8_e4m3fn), (v, "v", torch.float8_e4m3fn), (k_scale, "k_scale", torch.float32),
                          (v_scale, "v_scale", torch.float32)):
        if not isinstance(t, torch.Tensor) or t.dtype is not want:
            raise TypeError("the cache's %s must be a %s tensor" % (name, want))
        if t.device != x.device:
            raise ValueError("the cache's %s is on %s, not on %s" % (name, t.device, x.device))
    shape = k.shape
    if len(shape) != 4 or v.shape != shape or k_scale.shape != shape[:3] or v_scale.shape != shape[:3]:
        raise ValueError("the cache's k and v must be (pages, key heads, places per page, dim), their scales the same without dim")
    pages, kv_heads, page_size, dim = shape
    if dim != x.shape[2] or kv_heads < 1 or page_size < 1:
        raise ValueError("the cache has shape %s, rows have dim %d" % (tuple(shape), x.shape[2]))
    page, head, place, step = k.stride()
    scale_page, scale_head, scale_step = k_scale.stride()
    if k.numel() and (v.stride() != k.stride() or v_scale.stride() != k_scale.stride()):
        raise ValueError("the cache's k and v, and their scales, must have equal strides")
    if (step != 1 and dim > 1) or (scale_step != 1 and page_size > 1):
        raise ValueError("the cache needs unit stride along dim, and its scales along the places")
    if offsets is None or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets must be a vector of the number of sequences + 1 values")
    if offsets.dtype is not torch.int32 and offsets.dtype is not torch.int64:
        raise TypeError("offsets must be int32 or int64")
    seqs = offsets.numel() - 1
    qo = _places(offsets, offsets, x.device, seqs + 1, "offsets")
    kl = _places(lengths, offsets, x.device, seqs, "lengths")
    if not isinstance(page_table, torch.Tensor) or page_table.dtype is not torch.int32:
        raise TypeError("page_table must be an int32 tensor")
    if page_table.device != x.device:
        raise ValueError("page_table is on %s, not on %s" % (page_table.device, x.device))
    if page_table.dim() != 2 or page_table.shape[0] != seqs or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table must be (%d, pages of a sequence) with unit stride along the pages" % seqs)
    width = page_table.shape[1]
    # (a stride of a single page, head or place means nothing)
    return L.Cache(dtype, kv_heads, dim, 1 if offsets.dtype is torch.int64 else 0, tokens, seqs, pages, page_size, k.data_ptr(), v.data_ptr(),
                   k_scale.data_ptr(), v_scale.data_ptr(), page if pages > 1 else 0, head if kv_heads > 1 else 0, place if page_size > 1 else 0,
                   scale_page if pages > 1 else 0, scale_head if kv_heads > 1 else 0, page_table.data_ptr(),
                   page_table.stride(0) if seqs > 1 else width, width, qo, kl)


def fuse_cache_write(k, v, cache, offsets, page_table, lengths, stream=None):
    """C: fuse_cache_write.  Writes the keys and values of new tokens, rounded to 8 bits with a scale per token and head, into a Cache.

    k, v: (tokens, key heads, dim), bfloat16 or float16; parts of one projection can be passed as they are.  offsets: the sequences' first new tokens
    and the end of the last one; lengths: their keys, the new ones among them (the last ones): a new token goes to the place of its key.
    page_table: (sequences, pages) int32, the pages of every sequence in order."""
    if k.dim() != 3:
        raise ValueError("k must be (tokens, heads, dim)")
    f = _cache(cache, k, k.shape[0], offsets, page_table, lengths)
    at_k, at_v = _heads_of(k, k, "k", None, f.kv_heads), _heads_of(v, k, "v", k.shape[0], f.kv_heads)

    def call(handle):
        _check(L.load().fuse_cache_write(f, *at_k, *at_v, handle))

    return _run(k.device, stream, call)


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
    f = _cache(cache, q, q.shape[0], offsets, page_table, lengths)
    n, heads, dim = q.shape
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.device != q.device):
        raise ValueError("lse must be a contiguous float32 tensor of shape %s on %s" % (tuple(q.shape[:2]), q.device))
    d = L.CacheQuery(*_heads_of(q, q, "q"), heads, 1 if causal else 0, dim ** -0.5 if scale is None else scale, _cap(cap),
                     None if slopes is None else _row(slopes, q, torch.float32, heads, "slopes"),
                     None if tree is None else _row(tree, q, torch.int64, n, "tree"))
    lib = L.load()

    def call(handle):
        l = torch.empty((n, heads), dtype=torch.float32, device=q.device) if lse is None else lse
        o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        at = _heads_of(o, q, "out", n, heads)
        nbytes = lib.fuse_attention_cache_bytes(f, d)
        ws = _workspace(nbytes, q.device) if nbytes else None
        _check(lib.fuse_attention_cache(f, d, *at, l.data_ptr(), ws.data_ptr() if nbytes else None, nbytes, handle))
        return o, l

    return _run(q.device, stream, call)
