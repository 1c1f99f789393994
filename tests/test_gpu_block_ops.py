"""Operators of a transformer block on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

import block_ref as R
import paper_1801_00829_amd as F

pytestmark = pytest.mark.gpu

DT = {"fp64": torch.float64, "fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rnd(g, shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std + mean).to(dtype)


def strided(t, pad):
    """The same matrix on the GPU with `pad` more columns between its rows."""
    big = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=t.dtype, device="cuda")
    view = big[:, :t.shape[1]]
    view.copy_(t)
    return view


# ------------------------------------------------------------------------------ norms ---

def block_case(seed, dtype, rows, cols, kind, post, gate, pre=True, pad=0, std=1.0, mean=0.0):
    g, t = gen(seed), DT[dtype]

    def weight():
        w = rnd(g, (cols,), t, 0.3, 1.0)
        return (w, rnd(g, (cols,), t, 0.2)) if kind == "layer" else w

    c = dict(x=rnd(g, (rows, cols), t, std, mean), z=rnd(g, (rows, cols), t, std, mean), post=weight() if post else None,
             pre=weight() if pre else None, dh=rnd(g, (rows, cols), t), dy=rnd(g, (rows, cols), t))
    shape = {None: None, "rowvec": (cols,), "colvec": (rows,), "matrix": (rows, cols)}[gate]
    c["gate"] = None if gate is None else (gate, rnd(g, shape, t, 0.5, 0.5))
    return c


def to_gpu(v, pad=0):
    if v is None or isinstance(v, str):
        return v
    if isinstance(v, tuple):
        return tuple(to_gpu(x, pad) for x in v)
    return strided(v, pad) if v.dim() == 2 and pad else v.cuda()


def big(v, leaf=False):
    if v is None or isinstance(v, str):
        return v
    if isinstance(v, tuple):
        return tuple(big(x, leaf) for x in v)
    return v.double().cpu().requires_grad_(leaf)


def first(v):
    return v[0] if isinstance(v, tuple) else v


def fp32_steps(cols, t):
    """Half steps of the arithmetic that a norm's result is off by, relative to its largest terms: eight columns in order, ten
    levels over a group of threads, up to four steps of columns, twice (statistics, then means of products), and some twenty
    operations per element; in fp64 for fp64."""
    return (2 * (8 * 4 + 10) + 20) * (F64 if t == torch.float64 else R.F32)


F64 = 2.0 ** -53
NORM_CASES = [
    # dtype, rows, cols, kind, post, gate, pad
    ("bf16", 1, 64, "rms", True, None, 0), ("bf16", 5, 4096, "rms", True, "rowvec", 0), ("fp16", 7, 512, "rms", True, "colvec", 8),
    ("fp32", 3, 1111, "layer", True, "matrix", 0), ("bf16", 6, 1, "layer", True, "rowvec", 0), ("bf16", 33, 130, "rms", False, "matrix", 3),
    ("fp64", 9, 777, "layer", True, "rowvec", 0), ("fp64", 4, 2048, "rms", True, "colvec", 2), ("fp32", 300, 96, "layer", True, "rowvec", 0),
    ("fp16", 2, 8192, "layer", True, "matrix", 0), ("bf16", 3, 8200, "rms", True, "rowvec", 0), ("fp32", 2, 20001, "layer", True, "rowvec", 0),
    ("bf16", 2, 32768, "rms", True, "colvec", 0), ("fp64", 2, 32768, "layer", False, None, 0), ("bf16", 1000, 264, "rms", True, "rowvec", 0),
    ("fp32", 17, 8, "rms", False, None, 0), ("bf16", 65, 1000, "layer", False, "colvec", 0),
]


def norm_id(c):
    return "-".join(str(x) for x in c)


@pytest.mark.parametrize("c", NORM_CASES, ids=norm_id)
def test_block_norm(c):
    dtype, rows, cols, kind, post, gate, pad = c
    d = block_case(1, dtype, rows, cols, kind, post, gate)
    t, scale = DT[dtype], 0.7
    h, y = F.fuse_block_norm(to_gpu(d["x"], pad), to_gpu(d["z"], pad), gate=to_gpu(d["gate"], pad), scale=scale, post=to_gpu(d["post"]),
                             pre=to_gpu(d["pre"]), kind=kind)
    assert F.last_kernel() == "block_norm_kernel"
    x, z = big(d["x"]), big(d["z"])
    rh, ry = R.block(x, z, big(d["gate"]), scale, big(d["post"]), big(d["pre"]), kind, 1e-6)
    n = fp32_steps(cols, t)
    top = x.abs() + (rh - x).abs().amax(1, keepdim=True) + 1.0
    R.within(h, rh, R.half_step(t) * rh.abs() + n * top, "h")
    w = big(first(d["pre"])).abs()
    b = big(d["pre"][1]).abs() if kind == "layer" else 0.0
    r = 1.0 / ((rh - (rh.mean(1, keepdim=True) if kind == "layer" else 0.0)).square().mean(1, keepdim=True) + 1e-6).sqrt()
    size = (rh.abs().amax(1, keepdim=True) + top.amax(1, keepdim=True)) * r * w + b
    R.within(y, ry, R.half_step(t) * ry.abs() + n * (2 * size + size.amax(1, keepdim=True)), "y")


@pytest.mark.parametrize("c", NORM_CASES, ids=norm_id)
def test_block_norm_backward(c):
    dtype, rows, cols, kind, post, gate, pad = c
    d = block_case(2, dtype, rows, cols, kind, post, gate)
    t, scale, eps = DT[dtype], 0.7, 1e-3
    got = F.fuse_block_norm_backward(to_gpu(d["dh"], pad), to_gpu(d["dy"], pad), to_gpu(d["x"], pad), to_gpu(d["z"], pad),
                                     gate=to_gpu(d["gate"], pad), scale=scale, post=to_gpu(d["post"]), pre=to_gpu(d["pre"]), kind=kind, eps=eps)
    ref = block_grads(d, kind, scale, eps)
    n = fp32_steps(cols, t)
    for name, value in got._asdict().items():
        assert (value is None) == (ref.get(name) is None), name
        if value is None:
            continue
        want, terms = ref[name], ref["terms_" + name]
        # sums over the rows: up to ceil(rows / 256) in order per block, then 16 partial sums, then 16 slices
        more = (rows // 256 + 64) * (F64 if t == torch.float64 else R.F32) if want.dim() == 1 and name != "dgate" or gate == "rowvec" else 0.0
        R.within(value, want, R.half_step(t) * want.abs() + (n + more) * terms, name)


def block_grads(d, kind, scale, eps):
    """Gradients by automatic differentiation in 64 bits, and the sizes of what is added up in each of them."""
    h, z, gate, post, pre = big(d["x"], True), big(d["z"], True), big(d["gate"], True), big(d["post"], True), big(d["pre"], True)
    dh, dy = big(d["dh"]), big(d["dy"])
    tup = lambda p: p if isinstance(p, tuple) else (p, None)  # noqa: E731
    out = {}
    y = R.norm(h, pre, kind, eps)
    leaves = [v for v in (h,) + tup(pre) if v is not None]
    got = torch.autograd.grad(y, leaves, dy)
    out["dx"], out["dpre"] = dh + got[0], got[1]
    out["dpre_bias"] = got[2] if kind == "layer" else None
    u = z if post is None else R.norm(z, post, kind, eps)
    if gate is not None:
        u = u * (gate[1][:, None] if gate[0] == "colvec" else gate[1])
    names = [(k, v) for k, v in (("dz", z), ("dgate", gate and gate[1]), ("dpost", tup(post)[0]), ("dpost_bias", tup(post)[1])) if v is not None]
    out.update(zip((k for k, _ in names), torch.autograd.grad(u, [v for _, v in names], scale * out["dx"])))

    def stat(v):
        c = v - v.mean(1, keepdim=True) if kind == "layer" else v
        r = 1.0 / (c.square().mean(1, keepdim=True) + eps).sqrt()
        return v.abs().amax(1, keepdim=True) * r + 1.0, r       # the largest normalised value, with the mean not yet taken off

    with torch.no_grad():
        rows_max = lambda v: v.abs().amax(1, keepdim=True)  # noqa: E731
        n, r = stat(h)
        w = tup(pre)[0]
        out["terms_dx"] = dh.abs() + 3 * r * rows_max(dy * w) * n * n
        t = scale * (out["terms_dx"] + out["dx"].abs())
        out["terms_dpre"], out["terms_dpre_bias"] = 3 * (dy.abs() * n * n).sum(0), dy.abs().sum(0)
        nz, rz = stat(z)
        pw, pb = (tup(post)[0], tup(post)[1]) if post is not None else (None, None)
        size_u = z.abs() if post is None else 3 * nz * nz * pw.abs() + (0 if pb is None else pb.abs())
        g = torch.ones_like(h) if gate is None else (gate[1][:, None] if gate[0] == "colvec" else gate[1]).abs().expand_as(h)
        du = t * g
        out["terms_dz"] = du if post is None else 3 * rz * rows_max(du * pw) * nz * nz
        if post is not None:
            out["terms_dpost"], out["terms_dpost_bias"] = 3 * (du * nz * nz).sum(0), du.sum(0)
        if gate is not None:
            both = 2 * t * size_u
            out["terms_dgate"] = {"rowvec": both.sum(0), "colvec": both.sum(1), "matrix": both}[gate[0]]
    return out


def test_block_norm_parts_alone():
    d = block_case(3, "fp32", 9, 200, "rms", True, "rowvec")
    x, z, pre, post = (to_gpu(d[k]) for k in ("x", "z", "pre", "post"))
    h, y = F.fuse_block_norm(x, pre=pre)                                    # a norm, no block
    assert h is x
    want = R.norm(big(d["x"]), big(d["pre"]), "rms", 1e-6)
    R.within(y, want, 64 * R.F32 * (1 + want.abs()) * 4, "y")
    h, y = F.fuse_block_norm(x, z, post=post)                               # a block, no norm behind it
    assert y is None
    want = big(d["x"]) + R.norm(big(d["z"]), big(d["post"]), "rms", 1e-6)
    R.within(h, want, 64 * R.F32 * (1 + want.abs()) * 4, "h")
    kept = h.clone()
    x2 = x.clone()
    again, _ = F.fuse_block_norm(x2, z, post=post, h=x2)                    # in place
    assert again is x2 and torch.equal(x2, kept)
    one = F.fuse_block_norm_backward(None, to_gpu(d["dy"]), x, pre=pre)
    two = F.fuse_block_norm_backward(torch.zeros_like(x), to_gpu(d["dy"]), x, pre=pre)
    assert torch.equal(one.dx, two.dx) and torch.equal(one.dpre, two.dpre) and one.dz is None and one.dgate is None
    only = F.fuse_block_norm_backward(to_gpu(d["dh"]), None, x, z, post=post)
    assert torch.equal(only.dx, to_gpu(d["dh"])) and only.dpre is None and only.dpost is not None


def test_block_norm_gradient_against_differences():
    d = block_case(4, "fp64", 3, 37, "layer", True, "rowvec")
    scale, step = 0.7, 1e-5
    args = {k: to_gpu(d[k]) for k in ("x", "z", "gate", "post", "pre")}
    dh, dy = to_gpu(d["dh"]), to_gpu(d["dy"])

    def value(a):
        h, y = F.fuse_block_norm(a["x"], a["z"], gate=a["gate"], scale=scale, post=a["post"], pre=a["pre"], kind="layer")
        return float((h * dh).sum() + (y * dy).sum())

    h, _ = F.fuse_block_norm(args["x"], args["z"], gate=args["gate"], scale=scale, post=args["post"], pre=args["pre"], kind="layer")
    got = F.fuse_block_norm_backward(dh, dy, h, args["z"], gate=args["gate"], scale=scale, post=args["post"], pre=args["pre"], kind="layer")
    for name, pick in (("dx", lambda a: a["x"]), ("dz", lambda a: a["z"]), ("dgate", lambda a: a["gate"][1]), ("dpost", lambda a: a["post"][0]),
                       ("dpost_bias", lambda a: a["post"][1]), ("dpre", lambda a: a["pre"][0]), ("dpre_bias", lambda a: a["pre"][1])):
        t, grad = pick(args).view(-1), getattr(got, name).view(-1)
        for i in (0, t.numel() // 2, t.numel() - 1):
            kept = float(t[i])
            t[i] = kept + step
            up = value(args)
            t[i] = kept - step
            down = value(args)
            t[i] = kept
            # central differences: third derivatives of a norm of normal rows are below 1e3, so step^2 * 1e3 and 1e-16 * |value| / step
            assert abs((up - down) / (2 * step) - float(grad[i])) <= 1e-6 * (1 + abs(float(grad[i]))), (name, i)


def test_block_norm_empty_and_special_rows():
    for rows in (0, 1):
        x = torch.zeros(rows, 40, dtype=torch.bfloat16, device="cuda")
        w = torch.ones(40, dtype=torch.bfloat16, device="cuda")
        h, y = F.fuse_block_norm(x, x.clone(), post=w, pre=w)
        assert h.shape == y.shape == (rows, 40) and not h.any() and not y.any()
        g = F.fuse_block_norm_backward(x, x, x, x, post=w, pre=w)
        assert not g.dx.any() and not g.dpre.any()
    # one bad row stays alone; eps = 0 on fewer rows than a block holds
    x = torch.randn(3, 64, device="cuda")
    x[1] = math.inf
    w = torch.ones(64, device="cuda")
    _, y = F.fuse_block_norm(x, pre=w, eps=0.0)
    assert y[1].isnan().all() and y[0].isfinite().all() and y[2].isfinite().all()
    g = F.fuse_block_norm_backward(None, torch.ones_like(y[::2]), x[::2], pre=w, eps=0.0)
    assert g.dx.isfinite().all() and g.dpre.isfinite().all()


# -------------------------------------------------------------------------- attention ---

def attn_case(seed, dtype, heads, kv_heads, dim, lens, key_lens=None, room=None, spare=0, packed=False):
    """lens: queries per sequence; key_lens: keys (None: the same); room: places of a cache; spare: rows behind the last sequence."""
    g, t = gen(seed), DT[dtype]
    ends = torch.tensor([0] + lens).cumsum(0)
    c = dict(offsets=ends.to(torch.int32), key_offsets=None, key_lengths=None)
    tokens = int(ends[-1]) + spare
    keys = tokens
    if key_lens is not None and room is None:
        c["key_offsets"] = torch.tensor([0] + key_lens).cumsum(0).to(torch.int32)
        keys = int(c["key_offsets"][-1]) + spare
    elif room is not None:
        c["key_offsets"] = (torch.arange(len(lens) + 1) * room).to(torch.int32)
        c["key_lengths"] = torch.tensor(key_lens, dtype=torch.int32)
        keys = room * len(lens) + spare
    if packed and key_lens is None:
        qkv = rnd(g, (tokens, heads + 2 * kv_heads, dim), t).cuda()
        c["q"], c["k"], c["v"] = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    else:
        c["q"], c["k"], c["v"] = (rnd(g, (n, h, dim), t).cuda() for n, h in ((tokens, heads), (keys, kv_heads), (keys, kv_heads)))
    c["dout"] = rnd(g, (tokens, heads, dim), t).cuda()
    return c


def offs(c, wide=False):
    return {k: None if c[k] is None else c[k].to(torch.int64 if wide else torch.int32).cuda() for k in ("offsets", "key_offsets", "key_lengths")}


ATTN_CASES = {
    "one": ("bf16", 1, 1, 64, [1]),
    "two_of_one": ("fp16", 4, 2, 128, [1, 1]),
    "tile": ("bf16", 2, 1, 128, [64]),
    "odd": ("bf16", 6, 2, 64, [37, 1, 130]),
    "none_between": ("fp16", 4, 4, 72, [5, 0, 200, 0]),
    "wide_group": ("bf16", 8, 1, 8, [65]),
    "group_3": ("fp16", 6, 2, 80, [129, 63]),
    "long": ("bf16", 4, 2, 128, [600, 257]),
    "seventy": ("bf16", 2, 2, 64, [1, 3, 0, 7, 33, 2, 64] * 10),
    "shared_by_8": ("bf16", 8, 1, 128, [700, 90, 0]),
    "shared_by_6": ("fp16", 6, 1, 80, [1, 801]),
    "thousands": ("bf16", 1, 1, 16, [1, 0, 2] * 1700),
    "dim_96": ("fp16", 2, 1, 96, [191]),
    "dim_104": ("bf16", 3, 1, 104, [150]),
    "dim_24": ("bf16", 2, 1, 24, [150, 20]),
}
CROSS_CASES = {
    "token": ("bf16", 8, 2, 128, [1, 1, 1], [1, 77, 300], 320),
    "token_one_head": ("fp16", 8, 1, 64, [1], [257], 512),
    "tokens_long": ("bf16", 4, 4, 128, [1, 1], [2500, 1300], 2560),
    "some": ("fp16", 4, 2, 64, [3, 16, 2], [40, 16, 100], None),
    "more_queries": ("bf16", 4, 2, 64, [50, 130], [20, 1], None),
    "no_keys": ("bf16", 4, 2, 128, [5, 3], [0, 9], None),
    "chunk": ("bf16", 4, 2, 128, [100, 64], [400, 1000], 1024),
    "chunk_long": ("fp16", 2, 1, 80, [40], [3000], None),
    "token_many_splits": ("bf16", 4, 1, 64, [1], [20000], None),
    "chunk_two_splits": ("bf16", 8, 2, 64, [900], [1500], None),
    "many": ("fp16", 16, 2, 128, [2] * 40, list(range(2, 162, 4)), 200),
}


def check_forward(c, causal=True, scale=None, wide=False):
    o = offs(c, wide)
    out, lse = torch.full_like(c["dout"], 7.0), torch.full(c["q"].shape[:2], 7.0, device="cuda")
    got = F.fuse_attention(c["q"], c["k"], c["v"], **o, causal=causal, scale=scale, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    ref, ref_lse, far, far_lse = R.attention(c["q"], c["k"], c["v"], c["offsets"], c["key_offsets"], c["key_lengths"], causal, scale)
    n = int(c["offsets"][-1])
    R.within(out[:n], ref[:n], far[:n], "out")
    R.within(lse[:n], ref_lse[:n], far_lse[:n], "lse")
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()       # rows of no sequence are left as they were
    return out, lse


def check_backward(c, out, lse, causal=True, scale=None, wide=False):
    o = offs(c, wide)
    d = [torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") for t in (c["q"], c["k"], c["v"])]
    F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **o, causal=causal, scale=scale, dq=d[0], dk=d[1], dv=d[2])
    ref = R.attention_grad(c["dout"], c["q"], c["k"], c["v"], out, lse, c["offsets"], c["key_offsets"], c["key_lengths"], causal, scale)
    for got, (want, far), name in zip(d, ref, ("dq", "dk", "dv")):
        mine = ~want.isnan().reshape(want.shape[0], -1).all(1)
        R.within(got[mine.cuda()], want[mine], far[mine], name)
        assert (got[~mine.cuda()] == 7.0).all(), name
    return d


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", sorted(ATTN_CASES))
def test_attention(name, causal):
    dtype, heads, kv_heads, dim, lens = ATTN_CASES[name]
    c = attn_case(11, dtype, heads, kv_heads, dim, lens, spare=3 if causal else 0, packed=causal)
    out, lse = check_forward(c, causal, wide=causal)
    check_backward(c, out, lse, causal, wide=causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", sorted(CROSS_CASES))
def test_attention_over_other_keys(name, causal):
    dtype, heads, kv_heads, dim, lens, keys, room = CROSS_CASES[name]
    c = attn_case(12, dtype, heads, kv_heads, dim, lens, keys, room, spare=2)
    out, lse = check_forward(c, causal)
    check_backward(c, out, lse, causal)


def test_attention_scales_and_large_scores():
    c = attn_case(13, "bf16", 2, 1, 64, [90])
    check_forward(c, scale=1.0)                                    # scores of +-30: maxima move a lot
    check_forward(c, scale=1e-4)
    c["q"].mul_(30.0)
    out, lse = check_forward(c)
    check_backward(c, out, lse)
    rising = torch.arange(90, device="cuda").to(torch.bfloat16)    # every key beats the one before it
    c["q"].fill_(1.0)
    c["k"].copy_(rising[:, None, None].expand_as(c["k"]))
    check_forward(c, scale=0.05)


def test_attention_masked_values_have_no_influence():
    """NaN and infinities in keys and values that a query does not see: the cache behind a sequence's end, and later tokens."""
    for bad in (math.nan, math.inf, -math.inf):
        for dtype, dim in (("bf16", 128), ("fp16", 72)):
            c = attn_case(14, dtype, 4, 2, dim, [1, 3], [30, 70], 96)
            for b, n in enumerate((30, 70)):
                c["k"][b * 96 + n:(b + 1) * 96] = bad
                c["v"][b * 96 + n:(b + 1) * 96] = bad
            out, lse = check_forward(c)
            assert out.isfinite().all()
            check_backward(c, out, lse)
            c = attn_case(15, dtype, 4, 2, dim, [150])
            clean, clean_lse = check_forward(c)
            kept = [t.clone() for t in check_backward(c, clean, clean_lse)]
            c["k"][100] = bad
            c["v"][100] = bad
            out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
            assert torch.equal(out[:100], clean[:100]) or out[:100].isfinite().all()
            ref, _, far, _ = R.attention(c["q"], c["k"], c["v"], c["offsets"])
            R.within(out[:100], ref[:100], far[:100], "out")
            dq, _, _ = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], clean, clean_lse, **offs(c))
            R.within(dq[:100], kept[0][:100].double(), kept[0][:100].double().abs() * R.half_step(DT[dtype]) * 2 + 0.05, "dq")
            assert dq[:100].isfinite().all()
            # a bad query, or gradient, of an early place reaches earlier keys only
            c = attn_case(16, dtype, 2, 1, dim, [150])
            out, lse = check_forward(c)
            c["dout"][40] = bad
            _, dk, dv = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
            assert dk[41:].isfinite().all() and dv[41:].isfinite().all()


def test_attention_one_bad_value_reaches_what_sees_it():
    """A value that is not finite: NaN or an infinity in its own dim of every query that sees it, and nowhere else."""
    for dtype, dim in (("fp16", 128), ("bf16", 40)):
        c = attn_case(19, dtype, 4, 2, dim, [210, 66])
        clean, lse = check_forward(c)
        c["v"][130, 1, 7] = math.inf
        ref, _, far, _ = R.attention(c["q"], c["k"], c["v"], c["offsets"])
        out, lse2 = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
        assert torch.equal(lse, lse2)
        hit = ~ref.isfinite()
        assert hit[130:210, 2:, 7].all() and int(hit.sum()) == 80 * 2
        assert (~out.isfinite()).cpu().equal(hit)
        R.within(out.cpu()[~hit], ref[~hit], far[~hit], "out")
        # gradients: a bad query reaches the keys it sees, a bad key the queries that see it
        c = attn_case(20, dtype, 2, 1, dim, [140])
        out, lse = check_forward(c)
        # what the bad value does not reach is the clean inputs' gradient within its bound, not to the bit: the sums of steps with
        # such a value run in another order than the matrix units', with other fp32 roundings, which the bound counts
        good = R.attention_grad(c["dout"], c["q"], c["k"], c["v"], out, lse, c["offsets"])
        c["k"][90, 0, 3] = math.nan
        dq, _, _ = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
        R.within(dq[:90], good[0][0][:90], good[0][1][:90], "dq")
        assert not dq[90:].isfinite().any()
        c["k"][90, 0, 3] = 0.0
        good = R.attention_grad(c["dout"], c["q"], c["k"], c["v"], out, lse, c["offsets"])       # of the keys as they are now
        c["q"][50, 1, 5] = math.inf
        _, dk, dv = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
        R.within(dk[51:], good[1][0][51:], good[1][1][51:], "dk")
        R.within(dv[51:], good[2][0][51:], good[2][1][51:], "dv")
        for t in (dk, dv):
            assert not t[:51].isfinite().all()


def test_attention_bad_values_where_rows_are_split():
    c = attn_case(22, "bf16", 8, 1, 64, [640])                     # the keys' gradients are sums of several blocks
    out, lse = check_forward(c)
    good = R.attention_grad(c["dout"], c["q"], c["k"], c["v"], out, lse, c["offsets"])
    c["dout"][300, 5, 9] = math.nan
    c["q"][301, 2, 1] = math.inf
    _, dk, dv = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
    R.within(dk[302:], good[1][0][302:], good[1][1][302:], "dk")
    R.within(dv[302:], good[2][0][302:], good[2][1][302:], "dv")
    assert not dv[:301].isfinite().all()


def test_attention_same_results_again_and_on_other_streams():
    c = attn_case(17, "bf16", 8, 2, 128, [300, 77])
    o = offs(c)
    out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **o)
    grads = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **o)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        out2, lse2 = F.fuse_attention(c["q"], c["k"], c["v"], **o, stream=stream)
        again = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out2, lse2, **o, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        assert all(torch.equal(x, y) for x, y in zip(grads, again))


def test_attention_offsets_that_say_too_much():
    """Offsets and lengths beyond the arrays are cut down; nothing outside is read or written."""
    c = attn_case(18, "bf16", 2, 1, 64, [40, 24])
    good, _ = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
    wild = torch.tensor([0, 40, 5000000], dtype=torch.int32, device="cuda")
    out, lse = F.fuse_attention(c["q"], c["k"], c["v"], wild)
    assert torch.equal(out, good)
    F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, wild)
    lens = torch.tensor([1 << 30, -5], dtype=torch.int32, device="cuda")
    out, _ = F.fuse_attention(c["q"], c["k"], c["v"], wild, key_offsets=wild, key_lengths=lens)
    assert torch.equal(out[:40], good[:40]) and (out[40:] == 0).all()


# -------------------------------------------------------------------------- gradients ---

CLIP_LISTS = {
    "one": [("fp32", (1,))], "small": [("fp64", (10, 784)), ("fp64", (10,)), ("fp64", (3, 5))],
    "mixed": [("bf16", (300, 257)), ("fp32", (1025,)), ("fp16", (77, 3)), ("fp64", (8192,)), ("bf16", (8193,)), ("fp32", (0,)), ("fp32", (7, 2049))],
    "many": [("bf16", (17 + i, 33)) for i in range(300)],
    "large": [("bf16", (5000, 4099)), ("fp32", (4099,))],
}


@pytest.mark.parametrize("name", sorted(CLIP_LISTS))
@pytest.mark.parametrize("clipped", [True, False])
def test_grad_clip(name, clipped):
    g = gen(21)
    grads = [rnd(g, shape, DT[t], 0.1) for t, shape in CLIP_LISTS[name]]
    dev = [t.cuda() for t in grads]
    total = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    cells = sum(t.numel() for t in grads)
    tol = total * (math.sqrt(cells) + 64) * F64                    # roundings of squares and sums, of random sign
    norm = F.fuse_grad_norm(dev)
    assert norm.dtype == torch.float64 and abs(float(norm) - total) <= tol
    top = total * (0.5 if clipped else 2.0)
    factor = min(1.0, top / (total + 1e-6))
    out = [torch.empty_like(t) for t in dev]
    assert float(F.fuse_grad_clip(dev, top, out=out)) == float(norm)
    for t, o, src in zip(grads, out, dev):
        want = t.double() * factor
        # the factor is rounded to the arithmetic's type, then the product, then the result
        R.within(o, want, want.abs() * (R.half_step(t.dtype) + 3 * (F64 if t.dtype == torch.float64 else R.F32) + 2 * tol / total) +
                 torch.finfo(t.dtype).smallest_normal * torch.finfo(t.dtype).eps, "clipped")
        assert torch.equal(src.cpu(), t)
    F.fuse_grad_clip(dev, top, norm=norm)                          # in place, with the norm from before
    assert all(torch.equal(a, b) for a, b in zip(dev, out))


def test_grad_clip_of_views_and_odd_places():
    base = torch.randn(4000, device="cuda", dtype=torch.float32)
    grads = [base[1:8], base[9:2000], base[2001:4000].view(1999)]
    turned = torch.randn(31, 40, device="cuda").t()
    before = [t.clone() for t in grads + [turned]]
    norm = F.fuse_grad_clip(grads + [turned], 1.0)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in before))
    assert abs(float(norm) - want) <= 1e-12 * want
    for t, b in zip(grads + [turned], before):
        R.within(t, b.double() / (want + 1e-6), b.double().abs().cpu() / want * 4 * R.F32, "view")
    assert base[0] == base[0] and base[8] == base[8]


def test_grad_clip_values_that_are_no_numbers():
    t = torch.ones(5, device="cuda")
    t[2] = math.nan
    assert math.isnan(float(F.fuse_grad_clip([t], 1.0))) and t.isnan().all()
    t = torch.ones(5, device="cuda")
    t[2] = math.inf
    assert math.isinf(float(F.fuse_grad_clip([t], 1.0))) and t[2].isnan() and (t[[0, 1, 3, 4]] == 0).all()
    t = torch.zeros(5, device="cuda")
    assert float(F.fuse_grad_clip([t, torch.empty(0, device="cuda")], 1.0)) == 0.0 and not t.any()
    assert float(F.fuse_grad_norm([torch.empty(0, device="cuda")])) == 0.0
    big_ = torch.full((3,), 3e38, device="cuda")
    assert abs(float(F.fuse_grad_norm([big_])) / (3e38 * math.sqrt(3.0)) - 1.0) < 1e-6     # squares beyond fp32


# ---------------------------------------------------------------- large, and at once ---

def test_attention_far_places():
    """Keys and queries behind 2^31 elements."""
    far, n, hk, hq, dim = 2200000, 100, 8, 16, 128
    g = gen(61)
    k, v = (torch.zeros(far + n, hk, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = attn_case(62, "bf16", hq, hk, dim, [3], [n])
    k[far:], v[far:] = c["k"], c["v"]
    off, key_off = (torch.tensor(x, dtype=torch.int64, device="cuda") for x in ([0, 0, 3], [0, far, far + n]))
    out, lse = F.fuse_attention(c["q"], k, v, off, key_offsets=key_off)
    ref, ref_lse, bound, bound_lse = R.attention(c["q"], c["k"], c["v"], c["offsets"], c["key_offsets"])
    R.within(out, ref, bound, "out")
    R.within(lse, ref_lse, bound_lse, "lse")
    dq, dk, dv = F.fuse_attention_backward(c["dout"], c["q"], k, v, out, lse, off, key_offsets=key_off)
    want = R.attention_grad(c["dout"], c["q"], c["k"], c["v"], out, lse, c["offsets"], c["key_offsets"])
    for got, (value, far_), name in ((dq, want[0], "dq"), (dk[far:], want[1], "dk"), (dv[far:], want[2], "dv")):
        R.within(got, value, far_, name)
    assert not dk[:far:1001].any() and not dv[:far:1001].any()
    del k, v, dk, dv
    far, hq = 600000, 32
    c = attn_case(63, "bf16", hq, hk, dim, [n])
    q = torch.zeros(far + n, hq, dim, dtype=torch.bfloat16, device="cuda")
    q[far:] = c["q"]
    off, key_off = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, far, far + n], [0, 0, n]))
    out, lse = F.fuse_attention(q, c["k"], c["v"], off, key_offsets=key_off)
    ref, _, bound, _ = R.attention(c["q"], c["k"], c["v"], c["offsets"])
    R.within(out[far:], ref, bound, "out")
    assert not out[:far:997].any() and (lse[:far:997] == -math.inf).all()
    torch.cuda.empty_cache()


def test_norm_and_clip_far_places():
    rows, cols = 540000, 4096                                      # 2.2e9 elements
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-5:] = rnd(gen(64), (5, cols), torch.bfloat16).cuda()
    w = rnd(gen(65), (cols,), torch.bfloat16, 0.2, 1.0).cuda()
    h, y = F.fuse_block_norm(x, x, post=w, pre=w)
    h5, y5 = F.fuse_block_norm(x[-5:].clone(), x[-5:].clone(), post=w, pre=w)
    assert torch.equal(h[-5:], h5) and torch.equal(y[-5:], y5) and not h[:-5:1009].any()
    got = F.fuse_block_norm_backward(x, x, h, x, post=w, pre=w)
    five = F.fuse_block_norm_backward(x[-5:], x[-5:], h5, x[-5:], post=w, pre=w)
    assert torch.equal(got.dx[-5:], five.dx) and torch.equal(got.dz[-5:], five.dz)
    # the other rows add zeros; sums of five terms of size ten at most in two orders (fp32: 2 * 5 * 10 * 2^-24), both rounded to bf16
    for a, b in ((got.dpre, five.dpre), (got.dpost, five.dpost)):
        R.within(a, b, b.double().cpu().abs() * 2.0 ** -7 + 100 * R.F32, "dw")
    del h, y, got
    norm = F.fuse_grad_clip([x], 1.0)
    total = math.sqrt(float(rnd(gen(64), (5, cols), torch.bfloat16).double().square().sum()))
    assert abs(float(norm) - total) <= 1e-12 * total
    assert abs(math.sqrt(float(x[-5:].double().square().sum())) - 1.0) < 2.0 ** -8       # clipped to 1, each cell rounded to bf16
    del x
    torch.cuda.empty_cache()


def test_calls_of_several_threads():
    import threading
    cases = [step_state(71 + i) for i in range(3)]
    want = [[t.clone() for t in step(s)] for s in cases]
    torch.cuda.synchronize()
    got, errors = [None] * 3, []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    got[i] = step(cases[i])
            stream.synchronize()
        except Exception as e:                                     # (looked at below, in the test's own thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


# ----------------------------------------------------------------------- all together ---

def step(s):
    """Forward and backward of the attention half of a block, and the clipping of its gradients."""
    _, y = F.fuse_block_norm(s["x"], pre=s["w_in"])
    qkv = (y @ s["w_qkv"]).view(y.shape[0], -1, s["dim"])
    hq, hk = s["heads"], s["kv_heads"]
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    out, lse = F.fuse_attention(q, k, v, s["offsets"])
    z = out.flatten(1) @ s["w_out"]
    h, y2 = F.fuse_block_norm(s["x"], z, gate=("rowvec", s["gate"]), scale=0.5, post=s["w_post"], pre=s["w_next"])
    b = F.fuse_block_norm_backward(s["dh"], s["dy"], h, z, gate=("rowvec", s["gate"]), scale=0.5, post=s["w_post"], pre=s["w_next"])
    d_w_out = out.flatten(1).t() @ b.dz
    dout = (b.dz @ s["w_out"].t()).view_as(out)
    dqkv = torch.empty_like(qkv)
    F.fuse_attention_backward(dout, q, k, v, out, lse, s["offsets"], dq=dqkv[:, :hq], dk=dqkv[:, hq:hq + hk], dv=dqkv[:, hq + hk:])
    d_w_qkv = y.t() @ dqkv.flatten(1)
    a = F.fuse_block_norm_backward(b.dx, dqkv.flatten(1) @ s["w_qkv"].t(), s["x"], pre=s["w_in"])
    grads = [a.dpre, d_w_qkv, d_w_out, b.dgate, b.dpost, b.dpre]
    norm = F.fuse_grad_clip(grads, 1.0)
    return [h, y2, a.dx, norm] + grads


def step_state(seed, t=torch.bfloat16):
    g = gen(seed)
    heads, kv_heads, dim, cols = 6, 2, 64, 192
    lens = [70, 1, 129]
    s = dict(heads=heads, kv_heads=kv_heads, dim=dim, x=rnd(g, (200, cols), t), dh=rnd(g, (200, cols), t), dy=rnd(g, (200, cols), t),
             w_qkv=rnd(g, (cols, (heads + 2 * kv_heads) * dim), t, cols ** -0.5), w_out=rnd(g, (heads * dim, cols), t, (heads * dim) ** -0.5))
    for name in ("w_in", "gate", "w_post", "w_next"):
        s[name] = rnd(g, (cols,), t, 0.2, 1.0)
    s["offsets"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in s.items()}


def test_training_step_of_a_block():
    s = step_state(31)
    got = step(s)
    leaves = {k: v.double().cpu().requires_grad_(v.is_floating_point()) if v.is_floating_point() else v.cpu()
              for k, v in s.items() if isinstance(v, torch.Tensor)}
    y = R.norm(leaves["x"], leaves["w_in"], "rms", 1e-6)
    qkv = (y @ leaves["w_qkv"]).view(200, -1, 64)
    outs = []
    for rows, _ in R.sequences(leaves["offsets"], None, None):
        for h in range(6):
            p = torch.softmax(R._scores(qkv[rows, h], qkv[rows, 6 + h // 3], 0.125, True), 1)
            outs.append(p @ qkv[rows, 8 + h // 3])
    out = torch.cat([torch.stack(outs[i * 6:i * 6 + 6], 1) for i in range(3)])
    h, y2 = R.block(leaves["x"], out.flatten(1) @ leaves["w_out"], ("rowvec", leaves["gate"]), 0.5, leaves["w_post"], leaves["w_next"], "rms", 1e-6)
    loss = (h * leaves["dh"].detach()).sum() + (y2 * leaves["dy"].detach()).sum()
    names = ["w_in", "w_qkv", "w_out", "gate", "w_post", "w_next"]
    want = torch.autograd.grad(loss, [leaves["x"]] + [leaves[n] for n in names])
    total = math.sqrt(sum(float(w.square().sum()) for w in want[1:]))
    want = [h, y2, want[0], torch.tensor([total])] + [w / total for w in want[1:]]
    want = [w.detach() for w in want]
    for g, w, name in zip(got, want, ["h", "y", "dx", "norm"] + names):
        # some twelve roundings to bf16 on the way of every value, each off by at most half a step: 12 * 2^-8 in the 2-norm
        err = float((g.double().cpu().view_as(w) - w).norm() / w.norm())
        assert err <= 12 * 2.0 ** -8, (name, err)


def test_first_calls_inside_a_capture():
    """Nothing has to be warmed up: calls of sizes and types that this process has not made are captured and replayed."""
    g = gen(51)
    q = rnd(g, (90, 5, 48), torch.float16).cuda()
    x, w = rnd(g, (7, 12000), torch.float16).cuda(), rnd(g, (12000,), torch.float16).cuda()
    off = torch.tensor([0, 90], dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = F.fuse_attention(q, q, q, off)
        h, y = F.fuse_block_norm(x, x, post=w, pre=w)
        grads = F.fuse_block_norm_backward(x, x, h, x, post=w, pre=w)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want = list(F.fuse_attention(q, q, q, off)) + list(F.fuse_block_norm(x, x, post=w, pre=w))
        want += [t for t in F.fuse_block_norm_backward(x, x, h, x, post=w, pre=w) if t is not None]
        assert all(torch.equal(a, b) for a, b in zip([out, lse, h, y] + [t for t in grads if t is not None], want))


def test_training_step_in_two_graphs():
    """Two steps captured on one stream, replayed in turn and at once on two streams, against the eager results."""
    states = [step_state(41), step_state(42)]
    eager = [[t.clone() for t in step(s)] for s in states]
    torch.cuda.synchronize()
    graphs, results = [], []
    for s in states:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(s)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(step(s))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for t in results[0] + results[1]:
            t.zero_()
        torch.cuda.synchronize()
        if turn % 2:
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
        else:
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for got, want in zip(results, eager):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        step(states[turn % 2])                                     # the program's own work between the replays
        torch.cuda.synchronize()
