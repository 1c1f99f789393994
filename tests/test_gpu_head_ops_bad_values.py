"""Operators on the heads of a projection on the GPU beside values that are not finite: what does not meet them is within its own bounds."""
import math

import pytest
import torch

import block_ref as R
import head_ref as H
import paper_1801_00829_amd as F
from test_gpu_head_ops import cache_case, trees

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
