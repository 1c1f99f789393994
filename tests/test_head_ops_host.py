"""Refusals of the operators on the heads of a projection, and their descriptors: no GPU is needed, nothing is launched."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_1801_00829_amd as F
from paper_1801_00829_amd import _lib as L
from paper_1801_00829_amd import head_ops as H
from test_block_ops_host import EINVAL, ESHAPE, EUNSUPPORTED, FAR, attn, attn_grads, refused


def test_descriptors_are_laid_out_like_the_header(tmp_path):
    pairs = [("fuse_rotary", L.Rotary, H._ROTARY), ("fuse_rotary_grads", L.RotaryGrads, H._ROTARY_GRADS), ("fuse_cache", L.Cache, H._CACHE),
             ("fuse_cache_query", L.CacheQuery, H._CACHE_QUERY), ("fuse_attn_shape", L.AttnShape, None)]
    lines = ['#include <stdio.h>', '#include "fuse.h"', "int main(void) {"]
    for name, cls, _ in pairs:
        lines.append('printf("%%zu", sizeof(%s));' % name)
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (name, f[0]) for f in cls._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    said = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, (name, cls, packed) in zip(said, pairs):
        want = [ctypes.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_]
        assert [int(x) for x in line.split()] == want, name
        if packed is None:
            continue
        assert packed.size == want[0], name
        values = []                                        # a different one in every field
        for field, kind in cls._fields_:
            values += [len(values) + 1 + i for i in range(kind._length_)] if hasattr(kind, "_length_") else [len(values) + 1]
        got = cls.from_buffer_copy(packed.pack(*values))
        flat = []
        for field, kind in cls._fields_:
            v = getattr(got, field)
            flat += list(v) if hasattr(kind, "_length_") else [v]
        assert [int(v) for v in flat] == values, name


# ------------------------------------------------------------- norms and rotary positions ---

def rotary(**kw):
    f = L.Rotary(dtype=2, heads=8, kv_heads=2, dim=64, pairs=0, axes=1, positions_are_64=0, sections=(32, 0, 0, 0), tokens=4, position_ld=4,
                 positions=FAR, freqs=FAR, q_weight=FAR, k_weight=FAR, eps=1e-6, q=FAR, k=FAR, q_token_ld=512, q_head_ld=64, k_token_ld=128,
                 k_head_ld=64)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


def rotary_grads(**kw):
    g = L.RotaryGrads(dq_out=FAR, dk_out=FAR, dq=FAR, dk=FAR, dq_weight=FAR, dk_weight=FAR, dq_out_token_ld=512, dq_out_head_ld=64,
                      dk_out_token_ld=128, dk_out_head_ld=64, dq_token_ld=512, dq_head_ld=64, dk_token_ld=128, dk_head_ld=64)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


ROTARY_REFUSALS = [
    (dict(dtype=5), EINVAL, "dtype"), (dict(heads=0), EINVAL, "heads"), (dict(kv_heads=-1), EINVAL, "kv_heads"), (dict(dim=63), EUNSUPPORTED, "dim"),
    (dict(dim=258, q_head_ld=300, q_token_ld=4000, k_head_ld=300, k_token_ld=600), EUNSUPPORTED, "dim"), (dict(pairs=2), EINVAL, "pairs"),
    (dict(axes=0), EINVAL, "axes"), (dict(axes=5), EINVAL, "axes"), (dict(sections=(0, 0, 0, 0)), ESHAPE, "sections"),
    (dict(sections=(33, 0, 0, 0)), ESHAPE, "sections"), (dict(axes=2, sections=(33, -1, 0, 0)), EINVAL, "sections"), (dict(tokens=-1), EINVAL, "tokens"),
    (dict(tokens=1 << 31), EUNSUPPORTED, "tokens"), (dict(heads=5000), EUNSUPPORTED, "heads"), (dict(positions=None), EINVAL, "positions"),
    (dict(freqs=None), EINVAL, "freqs"), (dict(positions=FAR + 2), EINVAL, "aligned"), (dict(positions=FAR + 4, positions_are_64=1), EINVAL, "aligned"),
    (dict(freqs=FAR + 4), EINVAL, "aligned"), (dict(axes=2, sections=(16, 16, 0, 0), position_ld=3), ESHAPE, "position_ld"),
    (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"), (dict(kv_heads=0), EINVAL, "k_weight"), (dict(q_weight=FAR + 1), EINVAL, "aligned"),
    (dict(q=None), EINVAL, "q"), (dict(k=FAR + 1), EINVAL, "k"), (dict(q_head_ld=63), ESHAPE, "q"), (dict(k_token_ld=63), ESHAPE, "k"),
    (dict(q_token_ld=1 << 41), EUNSUPPORTED, "q"),
]


@pytest.mark.parametrize("kw,code,word", ROTARY_REFUSALS, ids=[str(i) for i in range(len(ROTARY_REFUSALS))])
def test_qk_rotary_refuses(kw, code, word):
    lib, f, g = L.load(), rotary(**kw), rotary_grads()
    refused(lib.fuse_qk_rotary(ctypes.byref(f), FAR, 65536, 512, FAR, 65536, 512, None), code, word)
    refused(lib.fuse_qk_rotary_backward(ctypes.byref(f), ctypes.byref(g), FAR, 1 << 40, None), code, word)


def test_qk_rotary_refuses_results():
    lib, f = L.load(), rotary()
    call = lambda q=FAR, k=FAR, q_ld=512, k_ld=128: lib.fuse_qk_rotary(ctypes.byref(f), q, q_ld, 64, k, k_ld, 64, None)  # noqa: E731
    refused(call(q=None), EINVAL, "q_out")
    refused(call(k=None), EINVAL, "k_out")
    refused(call(q_ld=8), ESHAPE, "q_out")
    refused(call(k=FAR + 1), EINVAL, "k_out")
    refused(lib.fuse_qk_rotary(None, FAR, 512, 64, FAR, 128, 64, None), EINVAL, "rotary")
    need = lib.fuse_qk_rotary_backward_bytes(ctypes.byref(f))
    assert need > 0 and lib.fuse_qk_rotary_backward_bytes(ctypes.byref(rotary(q_weight=None, k_weight=None))) == 0
    assert lib.fuse_qk_rotary_backward_bytes(ctypes.byref(rotary(dim=63))) == 0

    def back(ws=FAR, nbytes=need, **kw):
        g = rotary_grads(**kw)
        return lib.fuse_qk_rotary_backward(ctypes.byref(f), ctypes.byref(g), ws, nbytes, None)

    refused(back(dq_out=None), EINVAL, "dq_out")
    refused(back(dk=None), EINVAL, "dk")
    refused(back(dk_head_ld=32), ESHAPE, "dk")
    refused(back(dq_weight=None), EINVAL, "dq_weight")
    refused(back(dk_weight=FAR + 1), EINVAL, "aligned")
    refused(back(ws=None), EINVAL, "workspace")
    refused(back(ws=FAR + 8), EINVAL, "workspace")
    refused(back(nbytes=need - 1), EINVAL, "workspace")
    refused(lib.fuse_qk_rotary_backward(ctypes.byref(f), None, FAR, need, None), EINVAL, "grads")


# ------------------------------------------------------------------------ cache in 8 bits ---

def cache(**kw):
    f = L.Cache(dtype=2, kv_heads=2, dim=64, offsets_are_64=0, tokens=4, seqs=2, pages=5, page_size=16, k=FAR, v=FAR, k_scale=FAR, v_scale=FAR,
                page_ld=2048, head_ld=1024, place_ld=64, scale_page_ld=32, scale_head_ld=16, table=FAR, table_ld=2, table_width=2, offsets=FAR,
                lengths=FAR)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


def query(**kw):
    q = L.CacheQuery(q=FAR, q_token_ld=512, q_head_ld=64, heads=8, causal=1, scale=0.1, cap=0.0)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


CACHE_REFUSALS = [
    (dict(dtype=9), EINVAL, "dtype"), (dict(dtype=1), EUNSUPPORTED, "dtype"), (dict(kv_heads=0), EINVAL, "kv_heads"), (dict(dim=60), EUNSUPPORTED, "dim"),
    (dict(dim=136), EUNSUPPORTED, "dim"), (dict(page_size=0), EINVAL, "page_size"), (dict(pages=-1), EINVAL, "counts"), (dict(tokens=-1), EINVAL, "counts"),
    (dict(tokens=1 << 31), EUNSUPPORTED, "tokens"), (dict(seqs=1 << 24), EUNSUPPORTED, "sequences"), (dict(table_width=1 << 27, table_ld=1 << 27), EUNSUPPORTED, "places"),
    (dict(offsets=None), EINVAL, "offsets"), (dict(lengths=None), EINVAL, "lengths"), (dict(table=None), EINVAL, "table"), (dict(table_ld=1), ESHAPE, "table"),
    (dict(v=None), EINVAL, "cache"), (dict(k_scale=None), EINVAL, "cache"), (dict(offsets=FAR + 2), EINVAL, "aligned"),
    (dict(lengths=FAR + 4, offsets_are_64=1), EINVAL, "aligned"), (dict(table=FAR + 2), EINVAL, "aligned"), (dict(v_scale=FAR + 2), EINVAL, "aligned"),
    (dict(k=FAR + 4), EUNSUPPORTED, "8 bytes"), (dict(place_ld=68), EUNSUPPORTED, "8 bytes"), (dict(place_ld=56), ESHAPE, "strides"),
    (dict(head_ld=0), ESHAPE, "strides"), (dict(page_ld=8), ESHAPE, "strides"), (dict(scale_page_ld=0), ESHAPE, "strides"),
    (dict(page_ld=1 << 41), EUNSUPPORTED, "2^40"), (dict(page_size=1 << 31, table_width=0), EUNSUPPORTED, "2^30"),
]


@pytest.mark.parametrize("kw,code,word", CACHE_REFUSALS, ids=[str(i) for i in range(len(CACHE_REFUSALS))])
def test_cache_refuses(kw, code, word):
    lib, f, q = L.load(), cache(**kw), query()
    refused(lib.fuse_cache_write(ctypes.byref(f), FAR, 512, 128, FAR, 512, 128, None), code, word)
    refused(lib.fuse_attention_cache(ctypes.byref(f), ctypes.byref(q), FAR, 512, 64, FAR, FAR, 1 << 40, None), code, word)
    assert lib.fuse_attention_cache_bytes(ctypes.byref(f), ctypes.byref(q)) == 0


QUERY_REFUSALS = [
    (dict(heads=0), EINVAL, "heads"), (dict(heads=7), ESHAPE, "kv_heads"), (dict(heads=4098), EUNSUPPORTED, "heads"), (dict(scale=0.0), EINVAL, "scale"),
    (dict(scale=float("nan")), EINVAL, "scale"), (dict(cap=-1.0), EINVAL, "cap"), (dict(cap=float("inf")), EINVAL, "cap"), (dict(cap=1e-9), EINVAL, "cap"),
    (dict(cap=float("nan")), EINVAL, "cap"), (dict(tree=FAR, causal=0), EINVAL, "tree"), (dict(tree=FAR, slopes=FAR), EINVAL, "tree"),
    (dict(tree=FAR + 4), EINVAL, "aligned"), (dict(slopes=FAR + 2), EINVAL, "aligned"), (dict(q=None), EINVAL, "q"), (dict(q=FAR + 8), EUNSUPPORTED, "q"),
    (dict(q_token_ld=516), EUNSUPPORTED, "q"), (dict(q_head_ld=56), ESHAPE, "q"),
]


@pytest.mark.parametrize("kw,code,word", QUERY_REFUSALS, ids=[str(i) for i in range(len(QUERY_REFUSALS))])
def test_attention_cache_refuses(kw, code, word):
    lib, f, q = L.load(), cache(), query(**kw)
    refused(lib.fuse_attention_cache(ctypes.byref(f), ctypes.byref(q), FAR, 512, 64, FAR, FAR, 1 << 40, None), code, word)
    assert lib.fuse_attention_cache_bytes(ctypes.byref(f), ctypes.byref(q)) == 0


def test_cache_refuses_rows_and_results():
    lib, f, q = L.load(), cache(), query()
    refused(lib.fuse_cache_write(None, FAR, 512, 128, FAR, 512, 128, None), EINVAL, "cache")
    refused(lib.fuse_cache_write(ctypes.byref(cache(tokens=1 << 28)), FAR, 512, 128, FAR, 512, 128, None), EUNSUPPORTED, "blocks")
    refused(lib.fuse_cache_write(ctypes.byref(f), None, 512, 128, FAR, 512, 128, None), EINVAL, "k")
    refused(lib.fuse_cache_write(ctypes.byref(f), FAR, 512, 128, FAR, 512, 32, None), ESHAPE, "v")
    refused(lib.fuse_cache_write(ctypes.byref(f), FAR, 512, 128, FAR + 2, 512, 128, None), EUNSUPPORTED, "v")
    read = lambda out=FAR, token=512, head=64, lse=FAR, ws=FAR, n=1 << 40, q=q, f=f: lib.fuse_attention_cache(  # noqa: E731
        ctypes.byref(f), ctypes.byref(q) if q else None, out, token, head, lse, ws, n, None)
    refused(read(q=None), EINVAL, "query")
    refused(read(out=None), EINVAL, "out")
    refused(read(token=8), ESHAPE, "out")
    refused(read(lse=FAR + 2), EINVAL, "lse")
    wide = cache(page_size=4096, place_ld=64, head_ld=1 << 18, page_ld=1 << 19)
    need = lib.fuse_attention_cache_bytes(ctypes.byref(wide), ctypes.byref(q))
    assert need > 0
    refused(read(f=wide, n=need - 1), EINVAL, "workspace")
    refused(read(f=wide, ws=None), EINVAL, "workspace")


# ------------------------------------------------------------- attention with shaped scores ---

SHAPE_REFUSALS = [(dict(cap=-2.0), EINVAL, "cap"), (dict(cap=1e-4), EINVAL, "cap"), (dict(cap=1.1e4), EINVAL, "cap"), (dict(cap=float("nan")), EINVAL, "cap"),
                  (dict(slopes=FAR + 1), EINVAL, "aligned"), (dict(prefix_lengths=FAR + 2), EINVAL, "aligned")]


@pytest.mark.parametrize("kw,code,word", SHAPE_REFUSALS, ids=[str(i) for i in range(len(SHAPE_REFUSALS))])
def test_shaped_attention_refuses(kw, code, word):
    lib, f, g, s = L.load(), attn(), attn_grads(), L.AttnShape(**kw)
    refused(lib.fuse_attention_shaped(ctypes.byref(f), ctypes.byref(s), FAR, 512, 64, FAR, FAR, 1 << 40, None), code, word)
    refused(lib.fuse_attention_shaped_backward(ctypes.byref(f), ctypes.byref(s), ctypes.byref(g), FAR, 1 << 40, None), code, word)
    assert lib.fuse_attention_shaped_backward_bytes(ctypes.byref(f), ctypes.byref(s)) == 0


def test_shaped_attention_refuses_what_attention_refuses():
    lib, s = L.load(), L.AttnShape(cap=30.0, prefix_lengths=FAR, slopes=FAR)
    f, g = attn(dim=60), attn_grads()
    refused(lib.fuse_attention_shaped(ctypes.byref(f), ctypes.byref(s), FAR, 512, 64, FAR, FAR, 1 << 40, None), EUNSUPPORTED, "dim")
    refused(lib.fuse_attention_shaped(ctypes.byref(attn(causal=0)), ctypes.byref(s), FAR, 512, 64, FAR, FAR, 1 << 40, None), EINVAL, "causal")
    refused(lib.fuse_attention_shaped(None, ctypes.byref(s), FAR, 512, 64, FAR, None, 0, None), EINVAL, "attn")
    f = attn()
    need = lib.fuse_attention_shaped_backward_bytes(ctypes.byref(f), ctypes.byref(s))
    assert need > lib.fuse_attention_backward_bytes(ctypes.byref(f))       # every row's place and slope
    assert lib.fuse_attention_shaped_backward_bytes(ctypes.byref(f), None) == lib.fuse_attention_backward_bytes(ctypes.byref(f))
    refused(lib.fuse_attention_shaped_backward(ctypes.byref(f), ctypes.byref(s), ctypes.byref(g), FAR, need - 1, None), EINVAL, "workspace")
    refused(lib.fuse_attention_shaped_backward(ctypes.byref(f), ctypes.byref(s), None, FAR, need, None), EINVAL, "grads")


# ------------------------------------------------------------------------------------ Python ---

def raises(kind, word, call):
    with pytest.raises(kind, match=word):
        call()


def test_python_rotary_refusals():
    q, k = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    pos, freqs, w = torch.zeros(4, dtype=torch.int32), torch.ones(32, dtype=torch.float64), torch.ones(64, dtype=torch.bfloat16)
    raises(ValueError, "CUDA", lambda: F.fuse_qk_rotary(q, k, pos, freqs))
    raises(ValueError, "CUDA", lambda: F.fuse_qk_rotary_backward(q, k, q, k, pos, freqs, q_weight=w))
    raises(TypeError, "float64, float32", lambda: F.fuse_qk_rotary(q.int(), k, pos, freqs))
    raises(ValueError, "tokens, heads, dim", lambda: F.fuse_qk_rotary(q[0], k, pos, freqs))
    raises(ValueError, "pairs", lambda: F.fuse_qk_rotary(q, k, pos, freqs, pairs="quarters"))
    raises(TypeError, "positions", lambda: F.fuse_qk_rotary(q, k, pos.float(), freqs))
    raises(TypeError, "freqs", lambda: F.fuse_qk_rotary(q, k, pos, freqs.float()))
    raises(ValueError, "positions", lambda: F.fuse_qk_rotary(q, k, pos[:3], freqs))
    raises(ValueError, "positions", lambda: F.fuse_qk_rotary(q, k, pos, freqs, sections=(16, 16)))
    raises(ValueError, "sections", lambda: F.fuse_qk_rotary(q, k, pos.expand(2, 4), freqs, sections=(16, 8)))
    raises(ValueError, "sections", lambda: F.fuse_qk_rotary(q, k, pos, freqs, sections=()))
    raises(ValueError, "unit stride along the tokens", lambda: F.fuse_qk_rotary(q, k, torch.zeros(4, 2, dtype=torch.int32).t(), freqs, sections=(16, 16)))
    raises(TypeError, "q_weight", lambda: F.fuse_qk_rotary(q, k, pos, freqs, q_weight=w.float()))
    raises(ValueError, "k_weight", lambda: F.fuse_qk_rotary(q, k, pos, freqs, k_weight=w[:32]))
    raises(ValueError, "k_weight", lambda: F.fuse_qk_rotary(q, None, pos, freqs, k_weight=w))
    raises(ValueError, "k_out", lambda: F.fuse_qk_rotary(q, None, pos, freqs, k_out=k))
    raises(TypeError, "k is", lambda: F.fuse_qk_rotary(q, k.float(), pos, freqs))
    raises(ValueError, "k has shape", lambda: F.fuse_qk_rotary(q, k[:2], pos, freqs))
    raises(ValueError, "unit stride", lambda: F.fuse_qk_rotary(q.transpose(1, 2)[:, :2], None, pos, freqs))
    raises(TypeError, "q must be a tensor", lambda: F.fuse_qk_rotary_backward(q, k, None, None, pos, freqs, q_weight=w))
    raises(ValueError, "dk needs keys", lambda: F.fuse_qk_rotary_backward(q, None, None, None, pos, freqs, dk=k))


def test_python_cache_refusals():
    c = F.cache_new(4, 16, 2, 64, device="cpu")
    assert c.k.shape == (4, 2, 16, 64) and c.k.dtype == torch.float8_e4m3fn and c.v_scale.shape == (4, 2, 16)
    k, q = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    off, table, lengths = torch.tensor([0, 1, 3], dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32), torch.tensor([1, 2], dtype=torch.int32)
    write = lambda k=k, v=k, c=c, off=off, table=table, lengths=lengths: F.fuse_cache_write(k, v, c, off, table, lengths)  # noqa: E731
    read = lambda q=q, c=c, off=off, table=table, lengths=lengths, **kw: F.fuse_attention_cache(q, c, off, table, lengths, **kw)  # noqa: E731
    for call in (write, read):
        raises(ValueError, "CUDA", call)
        raises(TypeError, "the cache's k ", lambda: call(c=c._replace(k=c.k.float())))
        raises(TypeError, "the cache's v_scale", lambda: call(c=c._replace(v_scale=c.v_scale.double())))
        raises(ValueError, "the cache's k and v must be", lambda: call(c=c._replace(v=c.v[:3])))
        raises(ValueError, "equal strides", lambda: call(c=c._replace(v_scale=c.v_scale.transpose(0, 1).contiguous().transpose(0, 1))))
        raises(TypeError, "page_table", lambda: call(table=table.long()))
        raises(ValueError, "page_table", lambda: call(table=table[:1]))
        raises(ValueError, "page_table", lambda: call(table=torch.zeros(2, 2, dtype=torch.int32).t()))
        raises(TypeError, "like offsets", lambda: call(lengths=lengths.long()))
        raises(ValueError, "lengths", lambda: call(lengths=lengths[:1]))
        raises(TypeError, "int32 or int64", lambda: call(off=off.float()))
    raises(ValueError, "k has shape", lambda: write(k=q))
    raises(ValueError, "v has shape", lambda: write(v=q))
    raises(ValueError, "rows have dim", lambda: write(k=k[..., :32]))
    raises(ValueError, "lse", lambda: read(lse=torch.zeros(2, 4)))
    raises(TypeError, "slopes", lambda: read(slopes=torch.zeros(4, dtype=torch.float64)))
    raises(ValueError, "slopes", lambda: read(slopes=torch.zeros(2)))
    raises(TypeError, "tree", lambda: read(tree=torch.zeros(3, dtype=torch.int32)))
    raises(ValueError, "tree", lambda: read(tree=torch.zeros(2, dtype=torch.int64)))
    raises(ValueError, "cap", lambda: read(cap=0.0))
    raises(ValueError, "cap", lambda: read(cap=float("nan")))


def test_python_shaped_attention_refusals():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    off, lse = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(4, 2)
    for call in (lambda **kw: F.fuse_attention(q, q, q, off, **kw), lambda **kw: F.fuse_attention_backward(q, q, q, q, q, lse, off, **kw)):
        raises(ValueError, "CUDA", lambda: call(cap=30.0, slopes=torch.zeros(2), prefix=off[1:]))
        raises(ValueError, "cap", lambda: call(cap=-1.0))
        raises(ValueError, "causal", lambda: call(prefix=off[1:], causal=False))
        raises(TypeError, "like offsets", lambda: call(prefix=off[1:].long()))
        raises(ValueError, "prefix", lambda: call(prefix=off))
        raises(TypeError, "slopes", lambda: call(slopes=off))
        raises(ValueError, "slopes", lambda: call(slopes=torch.zeros(3)))
