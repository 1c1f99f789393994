"""Operators on the heads of a projection on the GPU beside values that are not finite: what does not meet them is within its own bounds."""
import math

import pytest
import torch

import block_ref as R
import head_ref as H
import paper_1801_00829_amd as F
from test_gpu_block_ops import attn_case, offs
from test_gpu_head_ops import SHAPES, cache_case, on_gpu, shape_of, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("scale", [math.inf, math.nan])
def test_cache_scales_of_values_that_are_not_finite(dtype, scale):
    """They reach the results of who sees them, whose lse is a matter of keys alone."""
    for heads, kv_heads, dim, page, new, lengths, at in ((4, 2, 64, 16, [1], [40], 7), (4, 2, 128, 16, [6], [90], 86), (32, 2, 80, 24, [3], [700], 0),
                                                         (2, 1, 64, 64, [1], [9000], 4321), (8, 8, 96, 16, [40], [90], 89)):
        c = cache_case(67, dtype, heads, kv_heads, dim, page, new, lengths)
        tree = trees(8, new)
        (want, want_lse, far, far_lse), by_tree = H.cache_attention(c), H.cache_attention(c, tree=tree)
        c["cache"].v_scale[int(c["table"][0, at // page]), :, at % page] = scale
        meets = torch.arange(new[0]) + lengths[0] - new[0] >= at
        out, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
        R.within(lse, want_lse, far_lse, "lse")
        R.within(out.cpu()[~meets], want[~meets], far[~meets], "out")
        assert not out.cpu()[meets].isfinite().any()
        _, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"], tree=tree)
        R.within(lse, by_tree[1], by_tree[3], "lse")


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 72), ("fp16", 64)])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_shaped_gradients_beside_a_bad_key(shape, dtype, dim):
    """A key and its value that are not finite, given the results without them: gradients of the queries before it, and of all other keys and
    values, are those of the formula.  (A query that sees it has no gradient; every other key's, P o (dP - delta), does not hold it.)"""
    c = attn_case(15, dtype, 4, 2, dim, [150])
    s = shape_of(c, shape)
    if s["prefix"] is not None:
        s["prefix"] = torch.tensor([60], dtype=torch.int32)
    out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **on_gpu(s))
    (dq, far_q), (dk, far_k), (dv, far_v) = H.shaped_attention_grad(c, out, lse, **s)
    other = torch.arange(150) != 100
    for bad in (math.nan, math.inf, -math.inf):
        c["k"][100], c["v"][100] = bad, bad
        got = [t.cpu() for t in F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c), **on_gpu(s))]
        R.within(got[0][:100], dq[:100], far_q[:100], "dq")
        R.within(got[1][other], dk[other], far_k[other], "dk")
        R.within(got[2][other], dv[other], far_v[other], "dv")
