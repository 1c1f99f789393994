"""Transformer block's operators on the GPU where values are small, far apart or not finite, and in rows of no sequence.

Bounds here have no absolute term beyond what the type itself cannot hold: half a step of the result, fp16's subnormal one (2^-25)
where that is larger, and what the kernels say that they keep of the weights.
"""
import math

import pytest
import torch

import block_ref as R
import paper_1801_00829_amd as F
from test_gpu_block_ops import DT, attn_case, gen, offs, rnd

pytestmark = pytest.mark.gpu


def rounded(v, t):
    """How far a value of type t may be off by its own rounding."""
    return torch.clamp(R.half_step(t) * v.abs(), min=2.0 ** -25 if t == torch.float16 else 0.0)


def forward_bound(c, causal, scale):
    """(out, bound): weights are rounded to half a step of their own value, or in fp16 to 2^-36 of the row's sum where that is more."""
    t = c["q"].dtype
    ref = torch.zeros(c["q"].shape, dtype=torch.float64)
    far = torch.zeros_like(ref)
    q, k, v = (c[n].double().cpu() for n in "qkv")
    group = q.shape[1] // k.shape[1]
    for qs, ks in R.sequences(c["offsets"], c["key_offsets"], c["key_lengths"]):
        for h in range(q.shape[1]):
            qh, kh, vh = q[qs, h], k[ks, h // group], v[ks, h // group]
            s = R._scores(qh, kh, scale, causal)
            p = torch.softmax(s, 1)
            off = R._spread(qh, kh, scale)
            seen = (s != -math.inf).double()
            ref[qs, h] = p @ vh
            # (fp32 sums of the products: as many half steps as the matrix units add up in order, 16 at a time)
            e = R.half_step(t) + off + (kh.shape[0] // 16 + 16) * R.F32
            far[qs, h] = rounded(ref[qs, h], t) + 1.05 * e * (p @ vh.abs()) + (2.0 ** -36 * (seen @ vh.abs()) if t == torch.float16 else 0.0)
    return ref, far


# (score of a key whose value is 0, the other keys' values, number of keys, queries): the results are sums of small weights
SINKS = [(10.0, 1.0, 700, 40), (15.0, 1.0, 4096, 3), (16.0, 1.0, 4096, 40), (17.5, 1.0, 4097, 1), (17.5, 30.0, 300, 300), (19.0, 500.0, 1500, 70)]


@pytest.mark.parametrize("dtype,dim", [("fp16", 64), ("fp16", 128), ("fp16", 80), ("bf16", 64)])
@pytest.mark.parametrize("score,value,keys,queries", SINKS)
def test_attention_small_weights_beside_a_large_one(score, value, keys, queries, dtype, dim):
    g, t = gen(81), DT[dtype]
    for at in (0, keys // 2):                                      # the large weight comes first, or lifts the maximum later
        q, k = rnd(g, (queries, 4, dim), torch.float64, 0.3), rnd(g, (keys, 2, dim), torch.float64, 0.3 / math.sqrt(dim))
        v = rnd(g, (keys, 2, dim), torch.float64, 0.2, 1.0) * value
        q[:, :, 0], k[:, :, 0] = 1.0, 0.0
        k[at], v[at] = 0.0, 0.0
        k[at, :, 0] = score
        c = dict(q=q.to(t).cuda(), k=k.to(t).cuda(), v=v.to(t).cuda(), key_lengths=None,
                 offsets=torch.tensor([0, queries], dtype=torch.int32), key_offsets=torch.tensor([0, keys], dtype=torch.int32))
        for causal in (True, False):
            out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), causal=causal, scale=1.0)
            ref, far = forward_bound(c, causal, 1.0)
            R.within(out, ref, far, "out")
            _, want, _, far_lse = R.attention(c["q"], c["k"], c["v"], c["offsets"], c["key_offsets"], None, causal, 1.0)
            R.within(lse, want, far_lse, "lse")
