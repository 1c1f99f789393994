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


def gradients(c, out, lse, causal, scale):
    """((dq, bound), (dk, bound), (dv, bound)).  P and dS are rounded to half a step of their own values, or in fp16 to 2^-40 and to 2^-36 of
    the largest dS of the row (dq) or of the rows of all heads that share the key head (dk) where that is more."""
    t = c["q"].dtype
    sub = 1.0 if t == torch.float16 else 0.0
    dout, q, k, v, out, lse = (x.double().cpu() for x in (c["dout"], c["q"], c["k"], c["v"], out, lse))
    group, d = q.shape[1] // k.shape[1], q.shape[2]
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    fq, fk, fv = (torch.zeros_like(x) for x in (q, k, v))
    for qs, ks in R.sequences(c["offsets"], c["key_offsets"], c["key_lengths"]):
        n = (qs.stop - qs.start) * group
        if not n or ks.stop == ks.start:
            continue
        more = (max(n, ks.stop - ks.start) // 16 + 16) * R.F32
        for hk in range(k.shape[1]):
            kh, vh = k[ks, hk], v[ks, hk]
            found = []
            for h in range(hk * group, hk * group + group):
                s = R._scores(q[qs, h], kh, scale, causal)
                seen = (s != -math.inf).double()
                p = seen * torch.exp(s - lse[qs, h][:, None])
                off, size = R._spread(q[qs, h], kh, scale), (dout[qs, h] * out[qs, h]).abs().sum(1)[:, None]
                ds = p * (dout[qs, h] @ vh.T - (dout[qs, h] * out[qs, h]).sum(1)[:, None])
                fds = 1.05 * ((R.half_step(t) + off + more) * ds.abs() + p * (d + 8) * 2 * R.F32 * (dout[qs, h].abs() @ vh.abs().T + size))
                found.append((h, seen, p, ds, fds, off))
            top = max(float(x[3].abs().max()) for x in found)
            for h, seen, p, ds, fds, off in found:
                dq[qs, h] = scale * (ds @ kh)
                fq[qs, h] = scale * (fds + sub * 2.0 ** -36 * seen * ds.abs().amax(1, keepdim=True)) @ kh.abs()
                dk[ks, hk] += scale * (ds.T @ q[qs, h])
                fk[ks, hk] += scale * (fds + sub * 2.0 ** -36 * top * seen).T @ q[qs, h].abs()
                dv[ks, hk] += p.T @ dout[qs, h]
                fv[ks, hk] += 1.05 * ((R.half_step(t) + off + more) * p + sub * 2.0 ** -40 * seen).T @ dout[qs, h].abs()
    return (dq, fq + rounded(dq, t)), (dk, fk + rounded(dk, t)), (dv, fv + rounded(dv, t))


def check_gradients(c, causal=True, scale=None):
    scale = c["q"].shape[2] ** -0.5 if scale is None else scale
    out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), causal=causal, scale=scale)
    got = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c), causal=causal, scale=scale)
    for x, (want, far), name in zip(got, gradients(c, out, lse, causal, scale), ("dq", "dk", "dv")):
        R.within(x, want, far, name)
    return got


@pytest.mark.parametrize("dtype,heads,kv_heads,dim,lens", [("fp16", 2, 1, 128, [2048]), ("fp16", 4, 4, 64, [701, 0, 300]), ("fp16", 3, 1, 80, [900]),
                                                           ("fp16", 16, 2, 64, [5] * 40), ("bf16", 2, 1, 128, [700])])
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4])
def test_attention_small_gradients(dtype, heads, kv_heads, dim, lens, size):
    for causal in (True, False):
        c = attn_case(82, dtype, heads, kv_heads, dim, lens)
        c["dout"] = rnd(gen(83), c["dout"].shape, DT[dtype], size).cuda()
        check_gradients(c, causal)


def test_attention_large_gradients():
    """dS beyond fp16's range where dq, dk and dv are within it."""
    for dim, lens in ((64, [500, 3]), (128, [200])):
        c = attn_case(84, "fp16", 4, 2, dim, lens)
        c["v"].mul_(20.0)
        c["dout"].mul_(1000.0)
        got = check_gradients(c, scale=0.01)
        assert all(x.isfinite().all() for x in got)


def test_attention_gradients_of_different_sizes():
    """A few queries with gradients much larger than all the others': what does not see them keeps its digits."""
    c = attn_case(85, "fp16", 2, 1, 64, [900, 300])
    c["dout"].mul_(1e-3)
    c["dout"][[0, 1, 40, 899, 1000]] *= 1e4
    check_gradients(c)
    c["v"][500] *= 100.0                                           # one key with a value much larger than the others', met midway
    check_gradients(c)


@pytest.mark.parametrize("dtype,keys", [("bf16", 800), ("fp16", 1400), ("bf16", 2048), ("fp16", 2600)])
def test_attention_infinite_values_where_keys_are_split(dtype, keys):
    """An infinite value that all queries see, in the first, a middle or the last split, is an infinity in its own dim, whatever the splits."""
    c = attn_case(86, dtype, 4, 2, 72, [1], [keys])
    ref, _, far, _ = R.attention(c["q"], c["k"], c["v"], c["offsets"], c["key_offsets"])
    hit = torch.zeros(ref.shape, dtype=torch.bool)
    hit[:, 2:, 5] = True
    for at in (0, keys // 2, keys - 1):
        for bad in (math.inf, -math.inf):
            c["v"][at, 1, 5], kept = bad, float(c["v"][at, 1, 5])
            out = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))[0].cpu()
            c["v"][at, 1, 5] = kept
            assert (out[hit] == bad).all(), (at, bad)
            R.within(out[~hit], ref[~hit], far[~hit], "out")


def test_attention_results_do_not_depend_on_earlier_calls():
    """Results that are not finite send a block through its tiles again; what earlier kernels left in LDS has no say in that."""
    def before(value, t):
        x = torch.full((20000, 4, 128), value, dtype=t, device="cuda")
        off = torch.arange(0, 20001, 50, dtype=torch.int32, device="cuda")
        o, l = F.fuse_attention(x, x, x, off)
        F.fuse_attention_backward(x, x, x, x, o, l, off)

    for dtype, dim in (("bf16", 96), ("fp16", 96), ("bf16", 88), ("fp16", 128), ("bf16", 64)):
        c = attn_case(87, dtype, 8, 4, dim, [200, 130, 31] * 4)
        o = offs(c)
        out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **o)
        c["v"][::50, :, 3] = math.inf
        bad_q, bad_k = c["q"].clone(), c["k"].clone()
        bad_q[::70, :, 1] = math.inf
        bad_k[::90, :, 2] = math.nan
        found = []
        for value in (0.0, math.nan, 0.0, math.inf):
            before(value, DT[dtype])
            got = list(F.fuse_attention(c["q"], c["k"], c["v"], **o))
            before(value, DT[dtype])
            got += F.fuse_attention_backward(c["dout"], bad_q, bad_k, c["q"][:, :4].contiguous(), out, lse, **o)
            torch.cuda.synchronize()
            found.append([t.view(torch.int32 if t.dtype == torch.float32 else torch.int16) for t in got])
        for again in found[1:]:
            assert all(torch.equal(a, b) for a, b in zip(found[0], again)), (dtype, dim)


def covered(c):
    """Which queries, and which keys, belong to a sequence."""
    q, k = (torch.zeros(c[n].shape[0], dtype=torch.bool) for n in "qk")
    for qs, ks in R.sequences(c["offsets"], c["key_offsets"], c["key_lengths"]):
        q[qs], k[ks] = True, True
    return q.cuda(), k.cuda()


def stale(c):
    """Memory that the next allocations of these sizes will get, full of NaN."""
    kept = [torch.full_like(t, math.nan, memory_format=torch.contiguous_format) for t in (c["q"], c["k"], c["v"]) for _ in range(3)]
    torch.cuda.synchronize()
    del kept


REST_CASES = {
    # type, heads, kv_heads, dim, lengths, key lengths, room, spare rows; the first sequence's start
    "padded": ("bf16", 6, 2, 64, [37, 1, 130], None, None, 25, 0),
    "begins_late": ("fp16", 2, 1, 128, [70], None, None, 90, 17),
    "cache": ("bf16", 4, 4, 72, [1, 3, 0], [5, 96, 40], 96, 9, 0),
    "other_keys": ("fp16", 8, 1, 96, [9, 14], [100, 3], None, 3, 2),
    "many": ("bf16", 2, 2, 64, [1, 0, 3] * 700, [2, 1, 5] * 700, 8, 1, 0),
    "all_taken": ("bf16", 4, 2, 128, [64, 200], None, None, 0, 0),
    "long_gap": ("bf16", 3, 1, 24, [5], [7], 60000, 0, 0),
}


@pytest.mark.parametrize("name", sorted(REST_CASES))
def test_attention_gradients_of_no_sequence_are_zero(name):
    dtype, heads, kv_heads, dim, lens, keys, room, spare, late = REST_CASES[name]
    c = attn_case(88, dtype, heads, kv_heads, dim, lens, keys, room, spare=spare)
    if late:
        c["offsets"] += late
        if c["key_offsets"] is not None:
            c["key_offsets"] += late
    o, (in_q, in_k) = offs(c), covered(c)
    out, lse = torch.zeros_like(c["q"]), torch.zeros(c["q"].shape[:2], device="cuda")
    F.fuse_attention(c["q"], c["k"], c["v"], **o, out=out, lse=lse)
    args = (c["dout"], c["q"], c["k"], c["v"], out, lse)
    kept = [torch.full_like(t, 7.0, memory_format=torch.contiguous_format) for t in (c["q"], c["k"], c["v"])]
    F.fuse_attention_backward(*args, **o, dq=kept[0], dk=kept[1], dv=kept[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        stale(c)
        got = F.fuse_attention_backward(*args, **o, stream=stream)
        torch.cuda.synchronize()
        for x, want, rows in zip(got, kept, (in_q, in_k, in_k)):
            assert torch.equal(x[rows], want[rows]) and not x[~rows].any()
            assert (want[~rows] == 7.0).all()
    stale(c)
    mine = torch.full_like(kept[1], 7.0)                           # some results given, some made by the call
    dq, dk, dv = F.fuse_attention_backward(*args, **o, dk=mine)
    assert dk is mine and (dk[~in_k] == 7.0).all() and not dq[~in_q].any() and not dv[~in_k].any()
    assert torch.equal(dk[in_k], kept[1][in_k]) and torch.equal(dq[in_q], kept[0][in_q])


def test_attention_gradients_without_a_sequence():
    q = torch.ones(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(1, dtype=torch.int32, device="cuda")
    stale(dict(q=q, k=q, v=q))
    got = F.fuse_attention_backward(q, q, q, q, q, torch.zeros(5, 2, device="cuda"), off)
    assert not any(t.any() for t in got)


def test_attention_gradients_of_padded_batches_in_a_graph():
    """Offsets change between the replays of a captured call: what belongs to no sequence now is 0, whatever the replay before left there."""
    c = attn_case(89, "bf16", 4, 2, 64, [150, 50])
    off = c["offsets"].cuda()
    call = lambda: F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], *made, off)  # noqa: E731
    made = F.fuse_attention(c["q"], c["k"], c["v"], off)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for ends in ([0, 150, 200], [0, 20, 21], [30, 150, 190], [0, 150, 200]):
        off.copy_(torch.tensor(ends, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert not any(t[ends[-1]:].any() or t[:ends[0]].any() for t in got)


@pytest.mark.parametrize("dtype", ["fp64", "fp32", "bf16", "fp16"])
@pytest.mark.parametrize("inplace", [True, False])
def test_grad_clip_writes_its_tensors_only(dtype, inplace):
    """Cells between views that are clipped, on every alignment and of every length around what the kernels move at once."""
    t = DT[dtype]
    base = rnd(gen(91), (60000,), t).cuda()
    spans, at = [], 1
    for n in (1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 31, 33, 100, 255, 257, 1023, 1025, 8191, 8193, 16385):
        for skip in (1, 2, 3):                                     # cells left free in front of a view
            if at + skip + n < 59000:
                spans.append((at + skip, n))
                at += skip + n
    free = torch.ones(60000, dtype=torch.bool)
    for first, n in spans:
        free[first:first + n] = False
    grads = [base[i:i + n] for i, n in spans]
    kept = base.clone()
    where = base if inplace else torch.full_like(base, 3.0)
    out = None if inplace else [where[i + 1:i + 1 + n] for i, n in spans]
    norm = F.fuse_grad_clip(grads, 1.0, out=out)
    total = math.sqrt(sum(float(kept[i:i + n].double().square().sum()) for i, n in spans))
    assert abs(float(norm) - total) <= 1e-12 * total
    if inplace:
        assert torch.equal(base[free.cuda()], kept[free.cuda()])
    else:
        moved = torch.cat([torch.ones(1, dtype=torch.bool), free[:-1]]).cuda()
        assert torch.equal(base, kept) and (where[moved] == 3.0).all()
    # the factor is rounded to the arithmetic's type, then the product, then the result
    steps = R.half_step(t) + 4 * (2.0 ** -53 if t == torch.float64 else R.F32) + 1e-12
    for i, (first, n) in enumerate(spans):
        want = kept[first:first + n].double().cpu() / (total + 1e-6)
        R.within(grads[i] if inplace else out[i], want, want.abs() * steps + (2.0 ** -25 if t == torch.float16 else 0.0), "clipped")


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 72), ("fp16", 96), ("bf16", 40)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_attention_gradients_beside_a_bad_key(dtype, dim, bad):
    """With the clean call's out and lse, a key that is not finite reaches its own gradients and those of the queries that see it: the others
    are the clean inputs' within their bounds."""
    c = attn_case(92, dtype, 4, 2, dim, [170])
    out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
    (dq, fq), (dk, fk), (dv, fv) = gradients(c, out, lse, True, dim ** -0.5)
    for names in ("k", "v", "kv"):
        kept = {n: c[n][100].clone() for n in names}
        for n in names:
            c[n][100] = bad
        got = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
        R.within(got[0][:100], dq[:100], fq[:100], "dq")
        others = torch.arange(170) != 100
        R.within(got[1].cpu()[others], dk[others], fk[others], "dk")
        R.within(got[2].cpu()[others], dv[others], fv[others], "dv")
        for n in names:
            c[n][100] = kept[n]


@pytest.mark.parametrize("dtype,dim", [("fp16", 64), ("fp16", 128), ("bf16", 64)])
@pytest.mark.parametrize("lens", [[20], [33, 64], [300]])
def test_attention_gradients_of_keys_beside_an_infinite_one(dtype, dim, lens):
    """All queries see a key whose value is infinite, so none of the sizes of their dS is a number to scale by."""
    c = attn_case(93, dtype, 4, 2, dim, lens)
    c["dout"].mul_(8.0)
    out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
    _, (dk, fk), (dv, fv) = gradients(c, out, lse, True, dim ** -0.5)
    bad = c["offsets"][:-1].long() + 1
    for value in (math.inf, -math.inf, math.nan):
        c["v"][bad.cuda(), :, 3] = value                           # (in one dim: dS is infinite and not NaN)
        _, got_k, got_v = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
        others = torch.ones(dk.shape[0], dtype=torch.bool)
        others[bad] = False
        R.within(got_k.cpu()[others], dk[others], fk[others], "dk")
        R.within(got_v.cpu()[others], dv[others], fv[others], "dv")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_heads_far_apart(dtype):
    """Heads one behind the other in a long cache, and queries and gradients laid out likewise: 38 million elements between two heads."""
    room, n, dim, t = 300000, 150, 128, DT[dtype]

    def laid(x):
        big = torch.zeros(x.shape[1], room, dim, dtype=t, device="cuda")
        big[:, 7:7 + n] = x.transpose(0, 1)
        return big.transpose(0, 1)

    c = attn_case(94, dtype, 4, 2, dim, [n])
    off = torch.tensor([7, 7 + n], dtype=torch.int64, device="cuda")
    near = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
    grads = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], *near, **offs(c))
    q, k, v, dout = (laid(c[x]) for x in ("q", "k", "v", "dout"))
    out, lse = torch.zeros_like(q), torch.zeros(room, 4, device="cuda")
    F.fuse_attention(q, k, v, off, out=out, lse=lse)
    assert torch.equal(out[7:7 + n], near[0]) and torch.equal(lse[7:7 + n], near[1])
    far = [torch.zeros_like(x) for x in (q, k, v)]
    F.fuse_attention_backward(dout, q, k, v, out, lse, off, dq=far[0], dk=far[1], dv=far[2])
    bounds = gradients(c, *near, True, dim ** -0.5)                # (which rows share a step differs, so sums may be in another order)
    for x, (want, bound), name in zip(far, bounds, ("dq", "dk", "dv")):
        R.within(x[7:7 + n], want, bound, name)
        assert not x[:7].any() and not x[7 + n:].any()
    assert torch.equal(far[0][7:7 + n], grads[0])
