"""Refusals of the transformer block's operators, and the descriptors' layout: no GPU is needed, nothing is launched."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_1801_00829_amd as F
from paper_1801_00829_amd import _lib as L

FAR = 1 << 20                                             # a pointer on 16 bytes that nothing may read

EINVAL, ESHAPE, EUNSUPPORTED = -1, -2, -7


def test_descriptors_are_laid_out_like_the_header(tmp_path):
    pairs = [("fuse_block", L.Block), ("fuse_block_grads", L.BlockGrads), ("fuse_attn", L.Attn), ("fuse_attn_grads", L.AttnGrads),
             ("fuse_tensor", L.Tensor)]
    lines = ['#include <stdio.h>', '#include "fuse.h"', "int main(void) {"]
    for name, cls in pairs:
        lines.append('printf("%%zu", sizeof(%s));' % name)
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (name, f[0]) for f in cls._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    said = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, (name, cls) in zip(said, pairs):
        want = [ctypes.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_]
        assert [int(x) for x in line.split()] == want, name


def refused(rc, code, word):
    assert rc == code, (rc, L.load().fuse_last_error())
    assert word in L.load().fuse_last_error().decode()


def block(**kw):
    b = L.Block(dtype=2, norm=0, rows=4, cols=64, eps=1e-6, scale=1.0, z=FAR, z_ld=64, pre_weight=FAR, gate_kind=-1)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


BLOCK_REFUSALS = [
    (dict(dtype=7), EINVAL, "dtype"), (dict(norm=2), EINVAL, "norm"), (dict(rows=-1), EINVAL, "rows"), (dict(cols=0), EINVAL, "cols"),
    (dict(cols=32769, z_ld=40000), EUNSUPPORTED, "32768"), (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"),
    (dict(z=None, post_weight=FAR), EINVAL, "z"), (dict(z=None, gate_kind=1, gate=FAR), EINVAL, "z"), (dict(pre_bias=FAR), EINVAL, "bias"),
    (dict(norm=1, post_bias=FAR), EINVAL, "weight"), (dict(gate_kind=3), EINVAL, "gate_kind"), (dict(gate_kind=2), EINVAL, "gate"),
    (dict(z_ld=63), ESHAPE, "z"), (dict(gate_kind=0, gate=FAR, gate_ld=8), ESHAPE, "gate"), (dict(gate_kind=1, gate=FAR, gate_ld=0), ESHAPE, "gate"),
]


@pytest.mark.parametrize("kw,code,word", BLOCK_REFUSALS, ids=[str(i) for i in range(len(BLOCK_REFUSALS))])
def test_block_norm_refuses(kw, code, word):
    lib, b = L.load(), block(**kw)
    refused(lib.fuse_block_norm(ctypes.byref(b), FAR, 65536, FAR, 65536, FAR, 65536, None), code, word)
    g = L.BlockGrads(dx=FAR, dx_ld=65536)
    refused(lib.fuse_block_norm_backward(ctypes.byref(b), FAR, 65536, FAR, 65536, FAR, 65536, ctypes.byref(g), FAR, 1 << 40, None), code, word)


def test_block_norm_refuses_results():
    lib, b = L.load(), block()
    call = lambda x, h, y, ld=64: lib.fuse_block_norm(ctypes.byref(b), x, ld, h, ld, y, ld, None)  # noqa: E731
    refused(call(None, FAR, FAR), EINVAL, "x")
    refused(call(FAR, FAR, None), EINVAL, "y")
    refused(call(FAR, FAR, FAR, 60), ESHAPE, "x")
    b.pre_weight = None
    refused(call(FAR, None, None), EINVAL, "neither")
    refused(call(FAR, FAR, FAR), EINVAL, "y")
    b.z, b.pre_weight = None, FAR
    refused(call(FAR, FAR, FAR), EINVAL, "h")
    refused(lib.fuse_block_norm(None, FAR, 64, FAR, 64, FAR, 64, None), EINVAL, "block")
    assert lib.fuse_block_norm_backward_bytes(None) == 0 and lib.fuse_block_norm_backward_bytes(ctypes.byref(block(cols=40000))) == 0


def test_block_norm_backward_refuses():
    lib, b = L.load(), block()
    need = lib.fuse_block_norm_backward_bytes(ctypes.byref(b))
    assert need > 0

    def call(dh=FAR, dy=FAR, h=FAR, g=None, ws=FAR, nbytes=need, b=b):
        g = L.BlockGrads(dx=FAR, dx_ld=64) if g is None else g
        return lib.fuse_block_norm_backward(ctypes.byref(b), dh, 64, dy, 64, h, 64, ctypes.byref(g), ws, nbytes, None)

    refused(call(dh=None, dy=None), EINVAL, "dh")
    refused(call(h=None), EINVAL, "h")
    refused(call(ws=None), EINVAL, "workspace")
    refused(call(ws=FAR + 8), EINVAL, "workspace")
    refused(call(nbytes=need - 1), EINVAL, "workspace")
    refused(call(g=L.BlockGrads(dgate=FAR)), EINVAL, "gradient")
    refused(call(g=L.BlockGrads(dpost_weight=FAR)), EINVAL, "gradient")
    refused(call(g=L.BlockGrads(dx=FAR, dx_ld=8)), ESHAPE, "dx")
    refused(call(b=block(z=None), g=L.BlockGrads(dz=FAR, dz_ld=64)), EINVAL, "dz")
    refused(call(b=block(pre_weight=None)), EINVAL, "pre_weight")


def attn(**kw):
    f = L.Attn(dtype=2, heads=8, kv_heads=2, dim=64, causal=1, offsets_are_64=0, q_tokens=10, k_tokens=10, seqs=2, q_offsets=FAR, scale=0.1,
               q=FAR, k=FAR, v=FAR, q_token_ld=512, q_head_ld=64, k_token_ld=128, k_head_ld=64, v_token_ld=128, v_head_ld=64)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


ATTN_REFUSALS = [
    (dict(dtype=9), EINVAL, "dtype"), (dict(dtype=1), EUNSUPPORTED, "FUSE_BF16"), (dict(dim=0), EINVAL, "dim"), (dict(dim=60), EUNSUPPORTED, "dim"),
    (dict(dim=136), EUNSUPPORTED, "dim"), (dict(heads=7), ESHAPE, "kv_heads"), (dict(kv_heads=0), EINVAL, "kv_heads"), (dict(scale=0.0), EINVAL, "scale"),
    (dict(scale=-1.0), EINVAL, "scale"), (dict(scale=float("nan")), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale"),
    (dict(q_tokens=-1), EINVAL, "counts"), (dict(q_tokens=1 << 31), EUNSUPPORTED, "2^31"), (dict(q_offsets=None), EINVAL, "q_offsets"),
    (dict(k_tokens=11), ESHAPE, "k_offsets"), (dict(q_offsets=FAR + 2), EINVAL, "aligned"), (dict(offsets_are_64=1, k_lengths=FAR + 4), EINVAL, "aligned"),
    (dict(q=None), EINVAL, "q"), (dict(k=FAR + 8), EUNSUPPORTED, "k"), (dict(v_token_ld=132), EUNSUPPORTED, "v"), (dict(q_head_ld=32), ESHAPE, "q"),
    (dict(k_token_ld=8), ESHAPE, "k"), (dict(seqs=1 << 24), EUNSUPPORTED, "sequences"), (dict(seqs=1 << 23), EUNSUPPORTED, "tiles"),
]


@pytest.mark.parametrize("kw,code,word", ATTN_REFUSALS, ids=[str(i) for i in range(len(ATTN_REFUSALS))])
def test_attention_refuses(kw, code, word):
    lib, f = L.load(), attn(**kw)
    refused(lib.fuse_attention(ctypes.byref(f), FAR, 512, 64, FAR, FAR, 1 << 40, None), code, word)
    g = attn_grads()
    refused(lib.fuse_attention_backward(ctypes.byref(f), ctypes.byref(g), FAR, 1 << 40, None), code, word)


def attn_grads(**kw):
    g = L.AttnGrads(dout=FAR, out=FAR, lse=FAR, dq=FAR, dk=FAR, dv=FAR, dout_token_ld=512, dout_head_ld=64, out_token_ld=512, out_head_ld=64,
                    dq_token_ld=512, dq_head_ld=64, dk_token_ld=128, dk_head_ld=64, dv_token_ld=128, dv_head_ld=64)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def test_attention_refuses_results():
    lib, f = L.load(), attn()
    refused(lib.fuse_attention(None, FAR, 512, 64, FAR, None, 0, None), EINVAL, "attn")
    refused(lib.fuse_attention(ctypes.byref(f), None, 512, 64, FAR, FAR, 1 << 40, None), EINVAL, "out")
    refused(lib.fuse_attention(ctypes.byref(f), FAR, 512, 60, FAR, FAR, 1 << 40, None), EUNSUPPORTED, "out")
    refused(lib.fuse_attention(ctypes.byref(f), FAR, 512, 64, FAR + 2, FAR, 1 << 40, None), EINVAL, "lse")
    need = lib.fuse_attention_backward_bytes(ctypes.byref(f))
    assert need > 0
    for kw, code, word in ((dict(dout=None), EINVAL, "dout"), (dict(lse=None), EINVAL, "lse"), (dict(dk=None), EINVAL, "dk"),
                           (dict(dv_token_ld=4), EUNSUPPORTED, "dv"), (dict(dq_head_ld=56), ESHAPE, "dq"), (dict(out=FAR + 4), EUNSUPPORTED, "out")):
        g = attn_grads(**kw)
        refused(lib.fuse_attention_backward(ctypes.byref(f), ctypes.byref(g), FAR, need, None), code, word)
    g = attn_grads()
    refused(lib.fuse_attention_backward(ctypes.byref(f), ctypes.byref(g), FAR, need - 1, None), EINVAL, "workspace")
    refused(lib.fuse_attention_backward(ctypes.byref(f), None, FAR, need, None), EINVAL, "grads")


def tensors(*rows):
    arr = (L.Tensor * max(len(rows), 1))()
    for a, (data, out, count, dtype) in zip(arr, rows):
        a.data, a.out, a.count, a.dtype = data, out, count, dtype
    return arr, len(rows)


def test_grad_clip_refuses():
    lib = L.load()

    def clip(arr, n, top=1.0, eps=1e-6, norm_in=None, norm_out=FAR, ws=FAR, nbytes=1 << 30):
        return lib.fuse_grad_clip(arr, n, top, eps, norm_in, norm_out, ws, nbytes, None)

    one = tensors((FAR, None, 100, 1))
    assert lib.fuse_grad_norm_bytes(*one) == 8
    refused(clip(*one, top=-1.0), EINVAL, "max_norm")
    refused(clip(*one, top=float("nan")), EINVAL, "max_norm")
    refused(clip(*one, eps=-1.0), EINVAL, "eps")
    refused(clip(*one, norm_in=FAR), EINVAL, "norm_in")
    refused(clip(*one, norm_out=None), EINVAL, "norm_in")
    refused(clip(*one, nbytes=7), EINVAL, "workspace")
    refused(clip(None, 3), EINVAL, "tensors")
    refused(clip(*tensors((FAR, None, 10, 4))), EINVAL, "dtype")
    refused(clip(*tensors((None, None, 10, 1))), EINVAL, "data")
    refused(clip(*tensors((FAR + 2, None, 10, 1))), EINVAL, "aligned")
    refused(clip(*tensors((FAR, None, 10, 1), (FAR, None, 10, 1))), EINVAL, "overlaps")          # twice in place
    refused(clip(*tensors((FAR, None, 10, 1), (FAR + 36, None, 10, 1))), EINVAL, "overlaps")
    refused(clip(*tensors((FAR, FAR + 4, 10, 1))), EINVAL, "overlaps")
    refused(clip(*tensors((FAR, FAR + 400, 10, 1), (FAR + 80, FAR + 404, 10, 1))), EINVAL, "overlaps")
    refused(clip(*tensors((FAR, FAR + 80, 10, 1), (FAR + 80, FAR + 400, 10, 1))), EINVAL, "overlaps")
    refused(lib.fuse_grad_norm(*one, None, FAR, 8, None), EINVAL, "norm")
    refused(lib.fuse_grad_norm(*one, FAR, None, 0, None), EINVAL, "workspace")
    assert lib.fuse_grad_norm_bytes(*tensors((FAR, None, -1, 1))) == 0
    # two lists of the size that one launch takes, and one cell more: a partial sum per block of each
    many = tensors(*[(FAR + 4096 * i, None, 7, 1) for i in range(257)])
    assert lib.fuse_grad_norm_bytes(*many) == 8 * 257


def test_python_refusals():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    off = torch.tensor([0, 4], dtype=torch.int32)
    for call in (lambda: F.fuse_block_norm(x, pre=x[0]), lambda: F.fuse_block_norm_backward(x, None, x),
                 lambda: F.fuse_attention(q, q, q, off), lambda: F.fuse_grad_norm([x]), lambda: F.fuse_grad_clip([x], 1.0)):
        with pytest.raises(ValueError, match="CUDA"):                      # a host tensor raises before anything is launched
            call()
    with pytest.raises(TypeError):
        F.fuse_block_norm(x.int(), pre=x[0])
    with pytest.raises(TypeError, match="pre weight"):
        F.fuse_block_norm(x, pre=x[0].float())
    with pytest.raises(ValueError, match="64 values"):
        F.fuse_block_norm(x, pre=x[0, :32])
    with pytest.raises(ValueError, match="unit column stride"):
        F.fuse_block_norm(torch.zeros(64, 4, dtype=torch.bfloat16).t(), pre=x[0])
    with pytest.raises(ValueError, match="gate"):
        F.fuse_block_norm(x, x, gate=("scalar", x[0]), pre=x[0])
    with pytest.raises(ValueError, match="kind"):
        F.fuse_block_norm(x, pre=x[0], kind="batch")
    with pytest.raises(ValueError, match="z"):
        F.fuse_block_norm(x, pre=x[0], h=x)
    with pytest.raises(ValueError, match="shape"):
        F.fuse_block_norm(x, x[:2], pre=x[0])
    with pytest.raises(TypeError, match="int32 or int64"):
        F.fuse_attention(q, q, q, off.float())
    with pytest.raises(TypeError, match="like offsets"):
        F.fuse_attention(q, q, q, off, key_offsets=off.long())
    with pytest.raises(ValueError, match="key_offsets"):
        F.fuse_attention(q, q, q, off, key_lengths=off[1:])
    with pytest.raises(ValueError, match="2 values"):
        F.fuse_attention(q, q, q, off, key_offsets=off[:1])
    with pytest.raises(ValueError, match="unit stride"):
        F.fuse_attention(torch.zeros(4, 64, 2, dtype=torch.bfloat16).transpose(1, 2), q, q, off)
    with pytest.raises(ValueError, match="v has shape"):
        F.fuse_attention(q, q, q[:3], off)
    with pytest.raises(ValueError, match="lse"):
        F.fuse_attention_backward(q, q, q, q, q, torch.zeros(2, 4), off)
    with pytest.raises(ValueError, match="gaps"):
        F.fuse_grad_norm([torch.zeros(4, 8)[:, :4]])
    with pytest.raises(ValueError, match="no tensors"):
        F.fuse_grad_norm([])
    with pytest.raises(ValueError, match="results"):
        F.fuse_grad_clip([x], 1.0, out=[])
    with pytest.raises(TypeError, match="result 0"):
        F.fuse_grad_clip([x], 1.0, out=[x.float()])


def test_attention_zero_rest_refuses():
    lib = L.load()
    call = lambda f, g: lib.fuse_attention_zero_rest(ctypes.byref(f), ctypes.byref(g) if g else None, None)  # noqa: E731
    refused(call(attn(), None), EINVAL, "grads")
    refused(call(attn(dim=60), attn_grads()), EUNSUPPORTED, "dim")
    refused(call(attn(), attn_grads(dv_token_ld=4)), EUNSUPPORTED, "dv")
    refused(call(attn(), attn_grads(dq_head_ld=56)), ESHAPE, "dq")
    refused(call(attn(), attn_grads(dk=FAR + 4)), EUNSUPPORTED, "dk")
    assert call(attn(), L.AttnGrads()) == 0                                # no result is asked for: nothing is launched


def test_grad_clip_refuses_a_norm_within_its_tensors():
    lib = L.load()

    def clip(rows, norm_in=None, norm_out=None):
        return lib.fuse_grad_clip(*tensors(*rows), 1.0, 1e-6, norm_in, norm_out, FAR + (1 << 19), 1 << 18, None)

    place, away = FAR, FAR + 4096
    for at in (FAR, FAR + 72):                                             # its first and its last cell
        refused(clip([(place, None, 10, 0)], norm_out=at), EINVAL, "norm")                     # written while it is read
        refused(clip([(place, None, 10, 0)], norm_in=at), EINVAL, "norm")                      # read while it is written
        refused(clip([(away, None, 3, 1), (away + 64, place, 10, 0)], norm_in=at), EINVAL, "norm")
        refused(clip([(place, away, 10, 0)], norm_out=at), EINVAL, "norm")
    refused(clip([(place, None, 10, 2)], norm_out=FAR + 16), EINVAL, "norm")
    refused(clip([(place, None, 10, 2)], norm_out=FAR + 1004), EINVAL, "aligned")
