"""Operators on the heads of a projection on the GPU, against their definitions in 64 bits."""
import math

import pytest
import torch

import block_ref as R
import head_ref as H
import paper_1801_00829_amd as F
from test_gpu_block_ops import DT, attn_case, gen, offs, rnd

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


# ------------------------------------------------------------------------ cache in 8 bits ---

def cache_case(seed, dtype, heads, kv_heads, dim, page, new, lengths, index=torch.int32, spare=2, pitch=0):
    """Sequences with `new` tokens each and `lengths` keys, on pages in any order; pitch: places of this many more bytes than dim."""
    g, t = gen(seed), DT[dtype]
    width = max([1] + [-(-n // page) for n in lengths])
    pages = len(new) * width + spare
    shape = (pages, kv_heads, page, dim + pitch)
    data = [(rnd(g, shape, torch.float32, 150.0).clamp_(-448, 448).to(torch.float8_e4m3fn).cuda())[..., :dim] for _ in range(2)]
    scales = [(torch.rand(shape[:3], generator=g) * 0.01 + 0.003).cuda() for _ in range(2)]
    ends = [0]
    for n in new:
        ends.append(ends[-1] + n)
    kv = rnd(g, (ends[-1], 2 * kv_heads, dim), t).cuda()
    return dict(cache=F.Cache(*data, *scales), page=page, q=rnd(g, (ends[-1], heads, dim), t).cuda(), k=kv[:, :kv_heads], v=kv[:, kv_heads:],
                table=torch.randperm(pages, generator=g)[:len(new) * width].view(len(new), width).to(torch.int32).cuda(),
                offsets=torch.tensor(ends, dtype=index).cuda(), lengths=torch.tensor(lengths, dtype=index).cuda())


def bits(t):
    """e4m3 as its bytes; also of a view with gaps"""
    return t.view(torch.uint8) if t.is_contiguous() else torch.stack([x.contiguous().view(torch.uint8) for x in t.unbind(0)])


def check_write(c):
    """Writes, and compares every place of the cache: the new ones with their definition, the others with what they were."""
    before = [t.clone() for t in c["cache"]]
    F.fuse_cache_write(c["k"], c["v"], c["cache"], c["offsets"], c["table"], c["lengths"])
    want = [before[0].cpu().double(), before[1].cpu().double(), before[2].cpu(), before[3].cpu()]
    offsets, pages = c["offsets"].tolist(), before[0].shape[0]
    for s, length in enumerate(c["lengths"].tolist()):
        n = offsets[s + 1] - offsets[s]
        for i in range(n):
            place = length - n + i
            if place < 0 or place >= c["table"].shape[1] * c["page"]:
                continue
            page = int(c["table"][s, place // c["page"]])
            if not 0 <= page < pages:
                continue
            for w, x in ((0, c["k"]), (1, c["v"])):
                values, scales = H.quantised(x[offsets[s] + i].double().cpu())
                want[w][page, :, place % c["page"]] = values
                want[w + 2][page, :, place % c["page"]] = scales.float()
    for got, w, name in zip(c["cache"], want, c["cache"]._fields):
        got = got.cpu().double()
        same = (got == w.double()) | (got.isnan() & w.double().isnan())
        assert bool(same.all()), (name, (~same).nonzero()[0].tolist(), float(got[~same][0]), float(w[~same][0]))


WRITE_CASES = [
    # heads of the cache, dim, page, new, lengths
    (1, 64, 16, [1], [1]), (8, 128, 16, [1] * 5, [1, 16, 17, 40, 33]), (2, 80, 24, [30, 0, 7], [30, 50, 24]), (4, 128, 64, [200, 13], [230, 13]),
    (3, 8, 1, [5, 9], [6, 9]), (1, 120, 7, [33], [40]), (2, 96, 1000, [300, 300], [300, 777]), (2, 40, 16, [9, 3], [4, 0]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i", range(len(WRITE_CASES)))
def test_cache_write(i, dtype):
    kv_heads, dim, page, new, lengths = WRITE_CASES[i]
    check_write(cache_case(i, dtype, kv_heads, kv_heads, dim, page, new, lengths, [torch.int32, torch.int64][i % 2]))


def check_cache_attention(c, **kw):
    got = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"], **kw)
    want = H.cache_attention(c, **kw)
    rows = ~want[1].isnan().all(1)
    R.within(got[0].cpu()[rows], want[0][rows], want[2][rows], "out")
    R.within(got[1].cpu()[rows], want[1][rows], want[3][rows], "lse")
    return got


READ_CASES = [
    # heads, kv_heads, dim, page, new, lengths
    (1, 1, 64, 16, [1], [1]), (8, 1, 64, 16, [1], [512]), (32, 8, 128, 16, [1] * 5, [1, 700, 33, 4001, 0]), (4, 4, 128, 64, [1, 1], [31, 2000]),
    (6, 2, 80, 24, [1, 0, 5], [300, 20, 129]), (12, 4, 96, 7, [3, 3], [3, 500]), (8, 2, 40, 1, [4], [37]), (5, 1, 120, 33, [17], [200]),
    (2, 2, 8, 16, [1, 2], [5, 100]), (16, 2, 128, 16, [40], [41]), (8, 8, 72, 128, [70, 2], [90, 1000]), (64, 1, 128, 256, [2], [3000]),
    (4, 2, 64, 16, [9, 4], [5, 0]),                       # fewer keys than new tokens: the first ones see nothing
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i", range(len(READ_CASES)))
def test_attention_cache(i, dtype):
    c = cache_case(100 + i, dtype, *READ_CASES[i], [torch.int32, torch.int64][i % 2])
    check_cache_attention(c)
    check_cache_attention(c, causal=False, scale=0.3)
    check_cache_attention(c, cap=2.5)
    slopes = (2.0 ** -torch.arange(1, READ_CASES[i][0] + 1, dtype=torch.float32) * 3).cuda()
    check_cache_attention(c, slopes=slopes)
    check_cache_attention(c, slopes=slopes, cap=30.0, causal=False)


def trees(seed, new):
    g, words = gen(seed), []
    for n in new:
        seen = []
        for i in range(n):
            up = seen[int(torch.randint(max(0, i - 5), i, (1,), generator=g))] if i else 0
            seen.append(up | (1 << i if i < 64 else 0))
        words += [x - (1 << 64) if x >> 63 else x for x in seen]
    return torch.tensor(words, dtype=torch.int64).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i", range(len(READ_CASES)))
def test_attention_cache_tree(i, dtype):
    c = cache_case(200 + i, dtype, *READ_CASES[i])
    tree = trees(i, READ_CASES[i][4])
    check_cache_attention(c, tree=tree)
    tree[::3] = 0                                         # these see none of the new tokens
    check_cache_attention(c, tree=tree, cap=10.0)


# ------------------------------------------------------------- attention with shaped scores ---

SHAPED_CASES = {
    "one": ("bf16", 1, 1, 64, [1]),
    "two_of_one": ("fp16", 4, 2, 128, [1, 1]),
    "odd": ("bf16", 6, 2, 64, [37, 1, 130]),
    "none_between": ("fp16", 4, 4, 72, [5, 0, 200, 0]),
    "wide_group": ("bf16", 8, 1, 8, [65]),
    "group_3": ("fp16", 6, 2, 80, [129, 63]),
    "long": ("bf16", 4, 2, 128, [600, 257]),
    "seventy": ("bf16", 2, 2, 64, [1, 3, 0, 7, 33, 2, 64] * 10),
    "shared_by_8": ("bf16", 8, 1, 128, [700, 90, 0]),
    "shared_by_6": ("fp16", 6, 1, 80, [1, 801]),
    "dim_96": ("fp16", 2, 1, 96, [191]),
    # other keys than queries: lengths of both, room of a cache
    "token": ("bf16", 8, 2, 128, [1, 1, 1], [1, 77, 300], 320),
    "tokens_long": ("fp16", 4, 4, 128, [1, 1], [2500, 1300], 2560),
    "more_queries": ("bf16", 4, 2, 64, [50, 130], [20, 1], None),
    "no_keys": ("bf16", 4, 2, 128, [5, 3], [0, 9], None),
    "chunk": ("bf16", 4, 2, 128, [100, 64], [400, 1000], 1024),
    "chunk_long": ("fp16", 2, 1, 80, [40], [3000], None),
}
SHAPES = {"cap": (2.5, False, False), "slopes": (None, True, False), "prefix": (None, False, True), "cap_prefix": (30.0, False, True),
          "slopes_prefix": (None, True, True), "all": (5.0, True, True)}


def shape_of(c, name, seed=5):
    """Arguments of a shape: for the call, and for the reference."""
    cap, sloped, prefixed = SHAPES[name]
    g, seqs = gen(seed), c["offsets"].numel() - 1
    slopes = 2.0 ** (-8.0 * torch.rand(c["q"].shape[1], generator=g)) if sloped else None
    longest = int((c["key_offsets"] if c["key_offsets"] is not None else c["offsets"]).diff().max())
    prefix = torch.randint(-1, longest + 3, (seqs,), generator=g, dtype=torch.int32) if prefixed else None
    if prefixed and seqs > 1:
        prefix[1] = 0
    return dict(cap=cap, slopes=slopes, prefix=prefix)


def on_gpu(shape, wide=False):
    prefix = shape["prefix"]
    return dict(cap=shape["cap"], slopes=None if shape["slopes"] is None else shape["slopes"].cuda(),
                prefix=None if prefix is None else prefix.to(torch.int64 if wide else torch.int32).cuda())


def check_shaped(c, shape, causal=True, scale=None, wide=False):
    out, lse = torch.full_like(c["dout"], 7.0), torch.full(c["q"].shape[:2], 7.0, device="cuda")
    F.fuse_attention(c["q"], c["k"], c["v"], **offs(c, wide), causal=causal, scale=scale, out=out, lse=lse, **on_gpu(shape, wide))
    ref, ref_lse, far, far_lse = H.shaped_attention(c, causal, scale, **shape)
    n = int(c["offsets"][-1])
    R.within(out[:n], ref[:n], far[:n], "out")
    R.within(lse[:n], ref_lse[:n], far_lse[:n], "lse")
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()       # rows of no sequence are left as they were
    d = [torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") for t in (c["q"], c["k"], c["v"])]
    F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c, wide), causal=causal, scale=scale, dq=d[0], dk=d[1], dv=d[2],
                              **on_gpu(shape, wide))
    want = H.shaped_attention_grad(c, out, lse, causal, scale, **shape)
    for got, (w, f), name in zip(d, want, ("dq", "dk", "dv")):
        mine = ~w.isnan().reshape(w.shape[0], -1).all(1)
        R.within(got[mine.cuda()], w[mine], f[mine], name)
        assert (got[~mine.cuda()] == 7.0).all(), name


@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("name", sorted(SHAPED_CASES))
def test_shaped_attention(name, shape):
    dtype, heads, kv_heads, dim, *rest = SHAPED_CASES[name]
    c = attn_case(13, dtype, heads, kv_heads, dim, *rest, spare=3)
    check_shaped(c, shape_of(c, shape), wide=heads == 4)
    if SHAPES[shape][2] is False:
        check_shaped(c, shape_of(c, shape), causal=False, scale=0.4)
