"""Loads libfuse.so with ctypes and declares the C ABI of include/fuse.h."""
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfuse.so")

MAX_SIDES = 8


class Dense(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64)]


class CsrDesc(ctypes.Structure):
    _fields_ = [("vals", ctypes.c_void_p), ("colidx", ctypes.c_void_p), ("rowptr", ctypes.c_void_p),
                ("rowptr_is64", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("nnz", ctypes.c_int64)]


class Side(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("m", Dense), ("scalar", ctypes.c_double),
                ("sp", ctypes.POINTER(CsrDesc))]


class Tok(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int32), ("arg", ctypes.c_int32), ("imm", ctypes.c_double)]


class Expr(ctypes.Structure):
    _fields_ = [("toks", ctypes.POINTER(Tok)), ("ntoks", ctypes.c_int32)]


class Block(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("norm", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("eps", ctypes.c_double), ("scale", ctypes.c_double), ("z", ctypes.c_void_p), ("z_ld", ctypes.c_int64),
                ("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p),
                ("gate_kind", ctypes.c_int32), ("gate", ctypes.c_void_p), ("gate_ld", ctypes.c_int64)]


class BlockGrads(ctypes.Structure):
    _fields_ = [("dx", ctypes.c_void_p), ("dx_ld", ctypes.c_int64), ("dz", ctypes.c_void_p), ("dz_ld", ctypes.c_int64),
                ("dgate", ctypes.c_void_p), ("dgate_ld", ctypes.c_int64), ("dpost_weight", ctypes.c_void_p),
                ("dpost_bias", ctypes.c_void_p), ("dpre_weight", ctypes.c_void_p), ("dpre_bias", ctypes.c_void_p)]


class Attn(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "heads", "kv_heads", "dim", "causal", "offsets_are_64")] + \
               [(n, ctypes.c_int64) for n in ("q_tokens", "k_tokens", "seqs")] + \
               [(n, ctypes.c_void_p) for n in ("q_offsets", "k_offsets", "k_lengths")] + [("scale", ctypes.c_double)] + \
               [(n, ctypes.c_void_p) for n in ("q", "k", "v")] + \
               [(n, ctypes.c_int64) for n in ("q_token_ld", "q_head_ld", "k_token_ld", "k_head_ld", "v_token_ld", "v_head_ld")]


class AttnGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dout", "out", "lse")] + \
               [(n, ctypes.c_int64) for n in ("dout_token_ld", "dout_head_ld", "out_token_ld", "out_head_ld")] + \
               [(n, ctypes.c_void_p) for n in ("dq", "dk", "dv")] + \
               [(n, ctypes.c_int64) for n in ("dq_token_ld", "dq_head_ld", "dk_token_ld", "dk_head_ld", "dv_token_ld", "dv_head_ld")]


class AttnShape(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_double), ("slopes", ctypes.c_void_p), ("prefix_lengths", ctypes.c_void_p)]


class Rotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "heads", "kv_heads", "dim", "pairs", "axes", "positions_are_64")] + \
               [("sections", ctypes.c_int32 * 4), ("tokens", ctypes.c_int64), ("position_ld", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("positions", "freqs", "q_weight", "k_weight")] + [("eps", ctypes.c_double)] + \
               [(n, ctypes.c_void_p) for n in ("q", "k")] + \
               [(n, ctypes.c_int64) for n in ("q_token_ld", "q_head_ld", "k_token_ld", "k_head_ld")]


class RotaryGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dq_out", "dk_out")] + \
               [(n, ctypes.c_int64) for n in ("dq_out_token_ld", "dq_out_head_ld", "dk_out_token_ld", "dk_out_head_ld")] + \
               [(n, ctypes.c_void_p) for n in ("dq", "dk")] + \
               [(n, ctypes.c_int64) for n in ("dq_token_ld", "dq_head_ld", "dk_token_ld", "dk_head_ld")] + \
               [(n, ctypes.c_void_p) for n in ("dq_weight", "dk_weight")]


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "kv_heads", "dim", "offsets_are_64")] + \
               [(n, ctypes.c_int64) for n in ("tokens", "seqs", "pages", "page_size")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + \
               [(n, ctypes.c_int64) for n in ("page_ld", "head_ld", "place_ld", "scale_page_ld", "scale_head_ld")] + \
               [("table", ctypes.c_void_p), ("table_ld", ctypes.c_int64), ("table_width", ctypes.c_int64), ("offsets", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p)]


class CacheQuery(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_token_ld", ctypes.c_int64), ("q_head_ld", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("scale", ctypes.c_double), ("cap", ctypes.c_double), ("slopes", ctypes.c_void_p),
                ("tree", ctypes.c_void_p)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int32)]


_lib = None


def load():
    """Returns the loaded library; raises if libfuse.so has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libfuse.so is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(or paper_1801_00829_amd/build.py) first")
    # Share the HIP runtime that PyTorch has loaded: device pointers and streams
    # are only meaningful inside one runtime instance.  Loading torch's copies of
    # the runtime and of hipRTC first makes libfuse's NEEDED entries resolve to them.
    import torch
    tlib = os.path.join(os.path.dirname(torch.__file__), "lib")
    for name in ("libamdhip64.so", "libhiprtc.so"):
        p = os.path.join(tlib, name)
        if os.path.exists(p):
            ctypes.CDLL(p, mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    vp, ci, i64p, dp = ctypes.c_void_p, ctypes.c_int, P(ctypes.c_int64), P(ctypes.c_double)
    lib.fuse_cell.argtypes = [P(Expr), P(Dense), P(Side), ci, ci, vp, vp]
    lib.fuse_magg.argtypes = [P(Expr), ci, P(Dense), P(Side), ci, vp, vp]
    lib.fuse_magg_noalloc.argtypes = [P(Expr), ci, P(Dense), P(Side), ci, vp, vp]
    lib.fuse_row.argtypes = [P(Expr), P(Dense), P(CsrDesc), P(Side), ci, ci, vp, vp]
    lib.fuse_outer.argtypes = [P(Expr), P(CsrDesc), P(Dense), P(Dense), P(Side), ci, ci, vp, vp]
    lib.fuse_cell_csr.argtypes = [P(Expr), P(CsrDesc), P(Side), ci, ci, vp, vp]
    lib.fuse_magg_csr.argtypes = [P(Expr), ci, P(CsrDesc), P(Side), ci, vp, vp]
    lib.fuse_prepare_cell_csr.argtypes = [P(Expr), P(CsrDesc), P(Side), ci, ci]
    lib.fuse_prepare_magg_csr.argtypes = [P(Expr), ci, P(CsrDesc), P(Side), ci]
    lib.fuse_prepare_cell.argtypes = [P(Expr), P(Dense), P(Side), ci, ci]
    lib.fuse_prepare_magg.argtypes = [P(Expr), ci, P(Dense), P(Side), ci]
    lib.fuse_prepare_row.argtypes = [P(Expr), P(Dense), P(CsrDesc), P(Side), ci, ci]
    lib.fuse_prepare_outer.argtypes = [P(Expr), P(CsrDesc), P(Dense), P(Dense), P(Side), ci, ci]
    lib.fuse_outer_left_pattern_bytes.argtypes = [P(CsrDesc)]
    lib.fuse_outer_left_pattern_bytes.restype = ctypes.c_size_t
    lib.fuse_outer_left_prepare.argtypes = [P(CsrDesc), vp, vp]
    lib.fuse_outer_left_prepare.restype = ci
    lib.fuse_outer_left_values.argtypes = [P(CsrDesc), vp, vp]
    lib.fuse_outer_left_values.restype = ci
    lib.fuse_outer_left.argtypes = [P(Expr), P(CsrDesc), vp, P(Dense), P(Dense), P(Side), ci, vp, vp]
    lib.fuse_outer_left.restype = ci
    lib.fuse_row_out_count.argtypes = [P(Expr), P(Dense), P(CsrDesc), P(Side), ci, ci, i64p]
    lib.fuse_row_out_count.restype = ci
    lib.fuse_check_csr.argtypes = [P(CsrDesc), vp]
    for f in (lib.fuse_check_csr, lib.fuse_cell_csr, lib.fuse_magg_csr, lib.fuse_prepare_cell_csr, lib.fuse_prepare_magg_csr,
              lib.fuse_cell, lib.fuse_magg, lib.fuse_magg_noalloc, lib.fuse_row, lib.fuse_outer, lib.fuse_prepare_cell,
              lib.fuse_prepare_magg, lib.fuse_prepare_row, lib.fuse_prepare_outer):
        f.restype = ci
    i64, f64, size = ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
    for name, args in (("fuse_block_norm", [P(Block), vp, i64, vp, i64, vp, i64, vp]),
                       ("fuse_block_norm_backward", [P(Block), vp, i64, vp, i64, vp, i64, P(BlockGrads), vp, size, vp]),
                       ("fuse_attention", [P(Attn), vp, i64, i64, vp, vp, size, vp]),
                       ("fuse_attention_backward", [P(Attn), P(AttnGrads), vp, size, vp]),
                       ("fuse_attention_shaped", [P(Attn), P(AttnShape), vp, i64, i64, vp, vp, size, vp]),
                       ("fuse_attention_shaped_backward", [P(Attn), P(AttnShape), P(AttnGrads), vp, size, vp]),
                       ("fuse_attention_zero_rest", [P(Attn), P(AttnGrads), vp]),
                       ("fuse_qk_rotary", [vp, vp, i64, i64, vp, i64, i64, vp]),
                       ("fuse_qk_rotary_backward", [vp, vp, vp, size, vp]),
                       ("fuse_cache_write", [vp, vp, i64, i64, vp, i64, i64, vp]),
                       ("fuse_attention_cache", [vp, vp, vp, i64, i64, vp, vp, size, vp]),
                       ("fuse_grad_norm", [vp, i64, vp, vp, size, vp]),
                       ("fuse_grad_clip", [vp, i64, f64, f64, vp, vp, vp, size, vp])):
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, ci
    for name, args in (("fuse_block_norm_backward_bytes", [P(Block)]), ("fuse_attention_bytes", [P(Attn)]),
                       ("fuse_attention_backward_bytes", [P(Attn)]), ("fuse_attention_shaped_backward_bytes", [P(Attn), P(AttnShape)]),
                        ("fuse_qk_rotary_backward_bytes", [vp]),
                       ("fuse_attention_cache_bytes", [vp, vp]), ("fuse_grad_norm_bytes", [vp, i64])):
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, size
    lib.fuse_last_error.restype = ctypes.c_char_p
    lib.fuse_last_kernel.restype = ctypes.c_char_p
    lib.fuse_cache_stats.argtypes = [i64p, i64p, dp]
    lib.fuse_cache_stats.restype = ci
    lib.fuse_cache_clear.restype = None
    lib.fuse_cache_disk_hits.argtypes = []
    lib.fuse_cache_disk_hits.restype = ctypes.c_int64
    lib.fuse_last_source.argtypes = [ctypes.c_char_p, ctypes.c_size_t]
    lib.fuse_last_source.restype = ctypes.c_size_t
    lib.fuse_probe_copy.argtypes = [vp, vp, ctypes.c_int64, ci, vp]
    lib.fuse_probe_copy.restype = ci
    lib.fuse_probe_read.argtypes = [vp, ctypes.c_int64, ci, vp, vp]
    lib.fuse_probe_read.restype = ci
    lib.fuse_probe_gather.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, vp, ctypes.c_int64, ci, vp, vp]
    lib.fuse_probe_gather.restype = ci
    _lib = lib
    return lib
