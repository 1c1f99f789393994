"""Operators on the heads of a projection: thin wrappers with the names of the C entry points (argument marshalling only)."""
from collections import namedtuple

import torch

from . import _lib as L
from .api import _check
from .block_ops import _dtype, _heads_of, _like, _run, _vector, _workspace

PAIRS = {"halves": 0, "neighbours": 1}

RotaryGrads = namedtuple("RotaryGrads", "dq dk dq_weight dk_weight")
"""Gradients of fuse_qk_rotary; None where the call had no such input."""


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
