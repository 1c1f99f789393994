"""Operators on the heads of a projection on the GPU, against their definitions in 64 bits."""
import math

import pytest
import torch

import block_ref as R
import head_ref as H
import paper_1801_00829_amd as F
from test_gpu_block_ops import DT, gen, rnd

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------- norms and rotary positions ---

ROTARY_CASES = [
    # tokens, heads, kv_heads, dim, pairs per axis, pairs, norm
    (1, 1, 1, 128, (64,), "halves", True), (1, 32, 8, 128, (64,), "halves", True), (7, 8, 2, 64, (32,), "neighbours", True),
    (300, 12, 4, 80, (10, 10, 10), "neighbours", True), (61, 5, 5, 80, (16,), "halves", True), (33, 6, 2, 96, (13, 7), "halves", False),
    (129, 3, 1, 2, (1,), "halves", True), (17, 2, 1, 6, (1, 1), "neighbours", True), (40, 7, 1, 256, (128,), "halves", True),
    (40, 7, 1, 256, (60, 0, 20, 20), "neighbours", True), (23, 4, 4, 254, (127,), "halves", True), (23, 4, 2, 130, (1,), "neighbours", False),
    (5000, 3, 1, 64, (32,), "halves", True), (4099, 2, 2, 40, (9, 9), "halves", True), (9, 40, 0, 128, (64,), "halves", True),
]


def rotary_case(seed, dtype, tokens, heads, kv_heads, dim, sections, pairs, norm, far=5000):
    g, t = gen(seed), DT[dtype]
    qkv = rnd(g, (tokens, heads + 2 * kv_heads, dim), t, 1.5).cuda()
    c = dict(q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads] if kv_heads else None, q_weight=None, k_weight=None, pairs=pairs,
             sections=sections if len(sections) > 1 else None)
    if norm:
        c["q_weight"] = rnd(g, (dim,), t, 0.3, 1.0).cuda()
        c["k_weight"] = rnd(g, (dim,), t, 0.3, 1.0).cuda() if kv_heads else None
    shape = (tokens,) if len(sections) == 1 else (len(sections), tokens)
    c["positions"] = torch.randint(-far, far, shape, generator=g, dtype=torch.int64).to([torch.int32, torch.int64][seed % 2]).cuda()
    half = sum(sections)
    c["freqs"] = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).cuda()
    c["dq_out"] = rnd(g, (tokens, heads, dim), t, 0.02).cuda()
    c["dk_out"] = rnd(g, (tokens, kv_heads, dim), t, 0.02).cuda() if kv_heads else None
    return c


def rotary_args(c):
    return dict(q_weight=c["q_weight"], k_weight=c["k_weight"], sections=c["sections"], pairs=c["pairs"])


def check_rotary(c, got, eps=1e-6):
    angle = H.angles(c["positions"], c["freqs"], c["sections"])
    for x, w, y, name in ((c["q"], c["q_weight"], got[0], "q"), (c["k"], c["k_weight"], got[1], "k")):
        if x is None:
            assert y is None
            continue
        big, bw = x.double().cpu(), None if w is None else w.double().cpu()
        assert y.dtype == x.dtype
        R.within(y, H.rotary(big, bw, angle, c["pairs"], eps), H.rotary_bound(big, bw, angle, c["pairs"], eps, x.dtype), name)


def check_rotary_grad(c, got, eps=1e-6):
    angle = H.angles(c["positions"], c["freqs"], c["sections"])
    for n in "qk":
        dy, x, w = c["d%s_out" % n], c[n], c[n + "_weight"]
        dx, dw = getattr(got, "d" + n), getattr(got, "d%s_weight" % n)
        if dy is None:
            assert dx is None and dw is None
            continue
        want = H.rotary_grad(dy.double().cpu(), None if w is None else x.double().cpu(), None if w is None else w.double().cpu(), angle,
                             c["pairs"], eps, dy.dtype)
        R.within(dx, *want[0], "d" + n)
        if w is None:
            assert dw is None
        else:
            R.within(dw, *want[1], "d%s_weight" % n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32", "fp64"])
@pytest.mark.parametrize("i", range(len(ROTARY_CASES)))
def test_qk_rotary(i, dtype):
    c = rotary_case(i, dtype, *ROTARY_CASES[i])
    check_rotary(c, F.fuse_qk_rotary(c["q"], c["k"], c["positions"], c["freqs"], **rotary_args(c)))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32", "fp64"])
@pytest.mark.parametrize("i", range(len(ROTARY_CASES)))
def test_qk_rotary_backward(i, dtype):
    c = rotary_case(i, dtype, *ROTARY_CASES[i])
    got = F.fuse_qk_rotary_backward(c["dq_out"], c["dk_out"], c["q"], c["k"], c["positions"], c["freqs"], **rotary_args(c))
    check_rotary_grad(c, got)
