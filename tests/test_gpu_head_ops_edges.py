"""Operators on the heads of a projection on the GPU: strides, places, values that are far apart or not finite, streams and graphs, and a run
of them together."""
import math

import pytest
import torch

import block_ref as R
import head_ref as H
import paper_1801_00829_amd as F
from test_gpu_block_ops import DT, attn_case, gen, offs, rnd
from test_gpu_head_ops import (SHAPES, cache_case, check_cache_attention, check_rotary, check_rotary_grad, check_shaped, check_write, on_gpu,
                               rotary_args, rotary_case, shape_of, trees)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------- norms and rotary positions ---

def test_qk_rotary_in_place_and_into_views():
    for dtype, dim in (("bf16", 128), ("fp16", 80), ("fp32", 64), ("bf16", 42)):
        c = rotary_case(40, dtype, 50, 6, 2, dim, (dim // 4,), "halves", True)
        want = [t.clone() for t in F.fuse_qk_rotary(c["q"], c["k"], c["positions"], c["freqs"], **rotary_args(c))]
        grads = F.fuse_qk_rotary_backward(c["dq_out"], c["dk_out"], c["q"], c["k"], c["positions"], c["freqs"], **rotary_args(c))
        # gradients in place of those of the results, and of the inputs
        both = torch.cat([c["dq_out"], c["dk_out"]], 1)
        got = F.fuse_qk_rotary_backward(both[:, :6], both[:, 6:], c["q"], c["k"], c["positions"], c["freqs"], dq=both[:, :6], dk=both[:, 6:],
                                        **rotary_args(c))
        assert all(torch.equal(a, b) for a, b in zip(got, grads)) and torch.equal(both[:, :6], grads.dq)
        # in place within the projection: its other columns stay
        qkv = torch.randn(50, 10, dim, device="cuda").to(DT[dtype])
        qkv[:, :6], qkv[:, 6:8] = c["q"], c["k"]
        rest = qkv[:, 8:].clone()
        F.fuse_qk_rotary(qkv[:, :6], qkv[:, 6:8], c["positions"], c["freqs"], q_out=qkv[:, :6], k_out=qkv[:, 6:8], **rotary_args(c))
        assert torch.equal(qkv[:, :6], want[0]) and torch.equal(qkv[:, 6:8], want[1]) and torch.equal(qkv[:, 8:], rest)
        # heads before tokens, places off 16 bytes, gaps behind rows
        room = torch.zeros(6 * 50 * (dim + 3) + 1, dtype=DT[dtype], device="cuda")[1:].view(6, 50, dim + 3)
        room[:, :, :dim] = c["q"].transpose(0, 1)
        out, _ = F.fuse_qk_rotary(room[:, :, :dim].transpose(0, 1), None, c["positions"], c["freqs"], q_weight=c["q_weight"], pairs=c["pairs"],
                                  q_out=room[:, :, :dim].transpose(0, 1))
        # (rows off 16 bytes are summed in another order: off by a rounding of the result at most, and the sums' own)
        R.within(out, want[0].double(), 2.02 * R.half_step(DT[dtype]) * want[0].double().abs() + 40 * R.F32 * want[0].double().abs().amax(-1, keepdim=True), "q")
        assert not room[:, :, dim:].any()


def test_qk_rotary_far_positions():
    """Angles keep their digits: positions up to 2^31, negative ones among them."""
    for dtype in ("fp32", "fp64"):
        c = rotary_case(41, dtype, 64, 3, 1, 64, (32,), "halves", True, far=2 ** 31 - 1)
        check_rotary(c, F.fuse_qk_rotary(c["q"], c["k"], c["positions"], c["freqs"], **rotary_args(c)))
        check_rotary_grad(c, F.fuse_qk_rotary_backward(c["dq_out"], c["dk_out"], c["q"], c["k"], c["positions"], c["freqs"], **rotary_args(c)))


def test_qk_rotary_turns_as_it_says():
    """A quarter turn exchanges the dims of a pair, no turn leaves them, whatever their values."""
    x = torch.arange(1, 9, dtype=torch.float32, device="cuda").view(1, 1, 8).repeat(3, 1, 1)
    freqs = torch.full((2,), math.pi / 2, dtype=torch.float64, device="cuda")
    at = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda")
    out, _ = F.fuse_qk_rotary(x, None, at, freqs)
    want = torch.tensor([[1, 2, 3, 4, 5, 6, 7, 8], [-3, -4, 1, 2, 5, 6, 7, 8], [3, 4, -1, -2, 5, 6, 7, 8]], dtype=torch.float64)
    R.within(out[:, 0], want, torch.full_like(want, 1e-6), "halves")
    out, _ = F.fuse_qk_rotary(x, None, at, freqs, pairs="neighbours")
    want = torch.tensor([[1, 2, 3, 4, 5, 6, 7, 8], [-2, 1, -4, 3, 5, 6, 7, 8], [2, -1, 4, -3, 5, 6, 7, 8]], dtype=torch.float64)
    R.within(out[:, 0], want, torch.full_like(want, 1e-6), "neighbours")
    # two axes: the first pair turns by the first row of positions, the second by the second
    out, _ = F.fuse_qk_rotary(x, None, torch.stack([at, 0 * at]), freqs, sections=(1, 1), pairs="neighbours")
    want[:, 2:4] = torch.tensor([3.0, 4.0])
    R.within(out[:, 0], want, torch.full_like(want, 1e-6), "axes")


def test_qk_rotary_same_positions_on_all_axes():
    c = rotary_case(45, "bf16", 30, 4, 2, 64, (10, 12, 10), "halves", True)
    at = c["positions"][1].clone()
    want = F.fuse_qk_rotary(c["q"], c["k"], at, c["freqs"], q_weight=c["q_weight"], k_weight=c["k_weight"])
    got = F.fuse_qk_rotary(c["q"], c["k"], at.expand(3, 30), c["freqs"], **rotary_args(c))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_qk_rotary_gradient_against_differences():
    c = rotary_case(42, "fp64", 5, 3, 2, 24, (4, 5), "neighbours", True)
    got = F.fuse_qk_rotary_backward(c["dq_out"], c["dk_out"], c["q"], c["k"], c["positions"], c["freqs"], eps=0.1, **rotary_args(c))

    def loss():
        q, k = F.fuse_qk_rotary(c["q"], c["k"], c["positions"], c["freqs"], eps=0.1, **rotary_args(c))
        return float((q * c["dq_out"]).sum() + (k * c["dk_out"]).sum())

    g, step = gen(43), 1e-5
    for name, grad in (("q", got.dq), ("k", got.dk), ("q_weight", got.dq_weight), ("k_weight", got.dk_weight)):
        for _ in range(8):
            at = tuple(int(torch.randint(0, n, (1,), generator=g)) for n in grad.shape)
            kept = float(c[name][at])
            c[name][at] = kept + step
            up = loss()
            c[name][at] = kept - step
            down = loss()
            c[name][at] = kept
            # central differences of a smooth function with derivatives of order one: step^2, and sums of some hundred terms of size 0.1 in 64 bits
            assert abs((up - down) / (2 * step) - float(grad[at])) <= 1e-8, name


def test_qk_rotary_empty_and_special_rows():
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    freqs = torch.ones(32, dtype=torch.float64, device="cuda")
    x = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    q, k = F.fuse_qk_rotary(x, x, none, freqs, q_weight=w, k_weight=w)
    assert q.shape == k.shape == (0, 4, 64)
    g = F.fuse_qk_rotary_backward(x, x, x, x, none, freqs, q_weight=w, k_weight=w)
    assert not g.dq_weight.any() and not g.dk_weight.any() and g.dq.shape == (0, 4, 64)
    # a row of zeros stays zeros with any eps but 0; a bad row stays alone
    x = torch.randn(3, 2, 64, device="cuda").to(torch.bfloat16)
    x[0, 0], x[1, 1, 5] = 0.0, math.inf
    at = torch.tensor([7, 8, 9], dtype=torch.int64, device="cuda")
    q, _ = F.fuse_qk_rotary(x, None, at, freqs, q_weight=w)
    assert not q[0, 0].any() and q[1, 1].isnan().any()
    q[1, 1] = 0.0
    assert q.isfinite().all()
    g = F.fuse_qk_rotary_backward(torch.ones_like(x), None, x, None, at, freqs, q_weight=w)
    assert g.dq[0].isfinite().all() and g.dq[1, 0].isfinite().all() and g.dq[2].isfinite().all() and g.dk is None and g.dk_weight is None
    # without a norm q and k are not read
    got = F.fuse_qk_rotary_backward(x, x, None, None, at, freqs)
    assert got.dq_weight is None and torch.equal(got.dq, got.dk)


def test_qk_rotary_many_tokens():
    """More tokens than blocks, and rows behind 2^31 elements."""
    n, heads, dim = 1100000, 16, 128
    q = torch.zeros(n, heads, dim, dtype=torch.bfloat16, device="cuda")
    g = gen(44)
    q[-7:] = rnd(g, (7, heads, dim), torch.bfloat16).cuda()
    w = rnd(g, (dim,), torch.bfloat16, 0.2, 1.0).cuda()
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    freqs = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    out, _ = F.fuse_qk_rotary(q, None, at, freqs, q_weight=w)
    few, _ = F.fuse_qk_rotary(q[-7:], None, at[-7:], freqs, q_weight=w)
    assert torch.equal(out[-7:], few) and not out[:-7:997].any()
    got = F.fuse_qk_rotary_backward(q, None, q, None, at, freqs, q_weight=w)
    few = F.fuse_qk_rotary_backward(q[-7:], None, q[-7:], None, at[-7:], freqs, q_weight=w)
    assert torch.equal(got.dq[-7:], few.dq) and not got.dq[:-7:997].any()
    # the other rows add zeros: sums of 112 terms of size 10 at most in two orders, both rounded
    R.within(got.dq_weight, few.dq_weight.double(), 2.0 ** -7 * few.dq_weight.double().abs() + 2 * 112 * 10 * 112 * R.F32, "dw")
    del q, out, got
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------ cache in 8 bits ---

def test_cache_write_rounds_to_nearest():
    """Every value of e4m3 and the middles between them, ties among them, beside a largest value of 448, in fp16 where they are exact."""
    values = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    middles = (values[1:] + values[:-1]) / 2
    all_ = torch.cat([values, middles, -values, -middles]).to(torch.float16)
    rows = -(-all_.numel() // 60)
    x = torch.zeros(rows, 1, 64, dtype=torch.float16)
    x.view(rows, 64)[:, :60].reshape(-1)[:] = 0
    flat = torch.zeros(rows * 60, dtype=torch.float16)
    flat[:all_.numel()] = all_
    x[:, 0, :60] = flat.view(rows, 60)
    x[:, 0, 63] = 448.0
    c = cache_case(50, "fp16", 1, 1, 64, 16, [rows], [rows])
    c["k"], c["v"] = x.cuda(), -x.cuda()
    check_write(c)


def test_cache_write_of_special_rows():
    for dtype in ("bf16", "fp16"):
        c = cache_case(51, dtype, 2, 2, 64, 16, [9], [9])
        k, v = c["k"].clone(), c["v"].clone()
        k[0], k[1, 0, 3], k[1, 1, 4], k[2, 0, 5] = 0.0, math.nan, math.inf, -math.inf
        v[3] *= 1e-4
        v[4] = torch.finfo(v.dtype).max
        v[5] = torch.finfo(v.dtype).tiny * (2.0 ** -3 if dtype == "fp16" else 1.0)
        v[6, 0, 1:], v[6, 1] = 0.0, -1.0
        c["k"], c["v"] = k, v
        check_write(c)
        page, at = int(c["table"][0, 0]), 0
        assert not c["cache"].k[page, :, at].float().any() and c["cache"].k_scale[page, 0, 1].isnan()


def test_cache_tables_that_say_too_much():
    """Pages that do not exist are not written, and others are read in their place; nothing outside is touched."""
    c = cache_case(52, "bf16", 4, 2, 64, 16, [20, 7], [40, 30])
    c["table"][0, 2], c["table"][1, 1] = -1, 1000000
    check_write(c)
    check_cache_attention(c)                               # (the reference reads the nearest page that exists, too)
    c["lengths"][0] = 1 << 30                              # all places of the table, and none of the new tokens
    check_cache_attention(c)
    c["lengths"][1] = -5
    out, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
    assert not out[20:].any() and (lse[20:] == -math.inf).all()
    wild = c["offsets"].clone()
    wild[2] = 1 << 30
    c["lengths"][1] = 30
    a = F.fuse_attention_cache(c["q"], c["cache"], wild, c["table"], c["lengths"])
    b = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # no pages at all, no places, no sequences, no tokens
    empty = F.cache_new(0, 16, 2, 64)
    for table in (c["table"], c["table"][:, :0]):
        F.fuse_cache_write(c["k"], c["v"], empty, c["offsets"], table, c["lengths"])
        out, lse = F.fuse_attention_cache(c["q"], empty, c["offsets"], table, c["lengths"])
        assert not out.any() and (lse == -math.inf).all()
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    for q in (c["q"], c["q"][:0]):
        F.fuse_cache_write(q[:, :2], q[:, 2:], c["cache"], none, c["table"][:0], none[:0])
        assert F.fuse_attention_cache(q, c["cache"], none, c["table"][:0], none[:0])[0].shape == q.shape


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_cache_of_sequences_that_outgrow_their_tables(dtype):
    """New tokens behind the table's last place are dropped, not written over older ones; the others stay where they belong."""
    c = cache_case(58, dtype, 6, 2, 64, 16, [5, 1, 20, 3], [40, 33, 45, 20])
    room = c["table"].shape[1] * 16                        # 48
    c["lengths"][:3] = torch.tensor([room + 2, room + 1, 5000], dtype=torch.int32)
    check_write(c)
    check_cache_attention(c)
    check_cache_attention(c, causal=False)
    check_cache_attention(c, slopes=torch.tensor([0.5, 0.25, 0.1, 0.0, 1.0, 0.01], device="cuda"))
    check_cache_attention(c, tree=torch.tensor([(2 << (i % 20)) - 1 for i in range(29)], device="cuda"))


def test_cache_rows_of_no_sequence():
    """Before the first and behind the last sequence nothing is read, written or answered."""
    c = cache_case(53, "fp16", 4, 2, 64, 16, [3, 5, 4], [20, 30, 10])
    off = c["offsets"][1:3].clone()
    c.update(offsets=off, lengths=c["lengths"][1:2], table=c["table"][1:2])
    c["k"], c["v"] = c["k"].clone(), c["v"].clone()
    c["k"][:3], c["v"][8:] = math.nan, math.nan
    check_write(c)
    c["q"][:3], c["q"][8:] = math.nan, math.nan
    out, lse = torch.full_like(c["q"], 7.0), torch.full((12, 4), 7.0, device="cuda")
    got = F.fuse_attention_cache(c["q"], c["cache"], off, c["table"], c["lengths"], out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    want = H.cache_attention(c)
    R.within(out[3:8], want[0][3:8], want[2][3:8], "out")
    R.within(lse[3:8], want[1][3:8], want[3][3:8], "lse")
    for t in (out, lse):
        assert (t[:3] == 7.0).all() and (t[8:] == 7.0).all()


@pytest.mark.parametrize("dim,page,pitch", [(128, 16, 32), (80, 24, 8), (64, 7, 16), (96, 16, 24)])
def test_cache_strides(dim, page, pitch):
    """Places with gaps between them, heads before pages, a table within a wider one, results with gaps."""
    c = cache_case(54, "bf16", 8, 2, dim, page, [2, 30], [70, 44], pitch=pitch)
    check_write(c)
    check_cache_attention(c)
    swapped = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (c["cache"].k_scale, c["cache"].v_scale)]
    data = [torch.empty(2, t.shape[0], page, dim, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).transpose(0, 1) for t in c["cache"][:2]]
    for to, t in zip(data, c["cache"][:2]):
        to.copy_(t)
    wide = torch.full((2, c["table"].shape[1] + 3), -7, dtype=torch.int32, device="cuda")
    wide[:, :c["table"].shape[1]] = c["table"]
    want = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
    c.update(cache=F.Cache(*data, *swapped), table=wide[:, :c["table"].shape[1]])
    out = torch.zeros(32, 9, dim, dtype=torch.bfloat16, device="cuda")
    got = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"], out=out[:, :8])
    R.within(got[0], want[0].double(), 2.02 * 2.0 ** -8 * want[0].double().abs() + 1e-5, "out")       # (another order of the same sums at most)
    assert not out[:, 8].any()
    check_write(c)
    check_cache_attention(c)


def test_cache_masked_places_have_no_influence():
    """Scales that are no number, and bytes that are none, in places that a query does not see."""
    for dtype, dim in (("bf16", 128), ("fp16", 72), ("fp16", 64)):
        for new, length in ((1, 50), (6, 50), (40, 90)):
            c = cache_case(55, dtype, 4, 2, dim, 16, [new], [length])
            good = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
            tree = trees(9, [new])
            good_tree = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"], tree=tree)
            place = length - 1                             # the last key: seen by the last query only
            page, at = int(c["table"][0, place // 16]), place % 16
            for what in ("k", "v", "k_scale", "v_scale"):
                kept = [t.clone() for t in c["cache"]]
                if what in "kv":
                    getattr(c["cache"], what).view(torch.uint8)[page, :, at, 3] = 0x7f
                    getattr(c["cache"], what).view(torch.uint8)[page, :, at, 5] = 0xff
                else:
                    getattr(c["cache"], what)[page, :, at] = math.nan
                for t in c["cache"][2:]:                   # behind the sequence, and on pages of none
                    t[page, :, at + 1:] = math.nan
                used = c["table"][0].tolist()
                for p in range(c["cache"].k.shape[0]):
                    if p not in used:
                        c["cache"].k_scale[p], c["cache"].v_scale[p] = math.nan, math.inf
                        c["cache"].v.view(torch.uint8)[p] = 0x7f
                out, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
                assert torch.equal(out[:-1], good[0][:-1]) and torch.equal(lse[:-1], good[1][:-1]), (what, new)
                assert out[-1].isnan().any() and (what in ("v", "v_scale") or lse[-1].isnan().any())
                out, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"], tree=tree)
                blind = (tree >> min(new - 1, 63)) & 1 == 0
                if new <= 64:
                    assert torch.equal(out[blind], good_tree[0][blind]) and out[~blind].isnan().any()
                for t, k in zip(c["cache"], kept):
                    t.view(torch.uint8).copy_(k.view(torch.uint8)) if t.dtype == torch.float8_e4m3fn else t.copy_(k)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_cache_scales_far_apart(dtype):
    """Values of very different sizes, zeros, and the smallest and large scales: the weights' digits follow what counts."""
    for seed, spread in ((56, 1.0), (57, 8.0), (58, 20.0)):
        c = cache_case(seed, dtype, 4, 2, 64, 16, [1, 5], [900, 300])
        g = gen(seed + 100)
        c["cache"].v_scale.mul_(torch.exp2(spread * torch.randn(c["cache"].v_scale.shape, generator=g).clamp(-3, 3)).cuda().mul_(0.25 if dtype == "fp16" else 1))
        c["cache"].v_scale.clamp_max_(2.0 if dtype == "fp16" else 1e30)
        c["cache"].v_scale[::3, :, ::5] = 0.0
        check_cache_attention(c)
    c = cache_case(59, dtype, 4, 2, 128, 16, [1], [333])
    c["cache"].v_scale.zero_()
    out, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
    assert not out.any()
    R.within(lse, H.cache_attention(c)[1], H.cache_attention(c)[3], "lse")
    c["cache"].v_scale.fill_(2.0 ** -100 / 448.0)
    check_cache_attention(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_cache_over_long_histories(dtype):
    """Up to the most splits that a call takes, joined by waves and by blocks, beside short sequences."""
    for heads, kv_heads, dim, page, new, lengths in ((8, 2, 128, 64, [1, 1, 1], [9000, 20, 0]), (4, 4, 64, 256, [1], [40000]), (6, 1, 72, 100, [3, 2], [7000, 5000]),
                                                     (32, 2, 96, 16, [2], [5003])):
        c = cache_case(66, dtype, heads, kv_heads, dim, page, new, lengths)
        check_cache_attention(c)
        check_cache_attention(c, tree=trees(3, new), cap=25.0)
        first = torch.full_like(c["q"], 7.0)               # rows of no sequence are not joined either
        off = (c["offsets"] - 1).clamp_min(0) if len(new) == 1 and new[0] > 1 else None
        if off is not None:
            want, _ = F.fuse_attention_cache(c["q"][:1].contiguous(), c["cache"], off, c["table"], c["lengths"])
            got, _ = F.fuse_attention_cache(c["q"], c["cache"], off, c["table"], c["lengths"], out=first)
            assert torch.equal(got[:1], want) and (got[1:] == 7.0).all()


def test_cache_of_keys_beyond_the_scores_range():
    """Scales of keys that no score holds: infinities where they are met, and 0 for a query of zeros."""
    c = cache_case(65, "bf16", 2, 1, 64, 16, [2], [50])
    c["q"][:, 0] = 0.0
    c["cache"].k_scale.fill_(1e38)
    out, lse = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"], scale=100.0)
    even = dict(c, q=c["q"][:, :1].clone(), cache=c["cache"]._replace(k_scale=torch.ones_like(c["cache"].k_scale)))
    want = H.cache_attention(even, scale=100.0)
    R.within(out[:, :1], want[0], want[2], "out")
    R.within(lse[:, :1], want[1], want[3], "lse")


def test_cache_far_places():
    """A cache of more than 2^32 bytes, and of pages further apart than that."""
    c = cache_case(60, "bf16", 8, 2, 128, 64, [2, 1], [300, 70])
    pages, shape = 40, (2, 64, 128)
    step = 600_000_000                                     # bytes between pages
    far = [torch.zeros(step * (pages - 1) + 2 * 64 * 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).as_strided((pages,) + shape, (step, 8192, 128, 1))
           for _ in range(2)]
    small, table = c["cache"], torch.randperm(pages, generator=gen(61))[:10].view(2, 5).to(torch.int32).cuda()
    scales = [torch.zeros(pages, 2, 64, device="cuda") for _ in range(2)]
    for s in range(2):
        for i in range(c["table"].shape[1]):
            for to, t in zip(far + scales, small):
                to[int(table[s, i])] = t[int(c["table"][s, i])]
    want = F.fuse_attention_cache(c["q"], small, c["offsets"], c["table"], c["lengths"])
    c.update(cache=F.Cache(*far, *scales), table=table)
    got = F.fuse_attention_cache(c["q"], c["cache"], c["offsets"], c["table"], c["lengths"])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check_write(dict(c, cache=F.Cache(*[t[:3] for t in c["cache"]]), table=torch.tensor([[2, 0, 1, 1, 1], [1, 1, 1, 1, 1]], dtype=torch.int32, device="cuda"),
                     lengths=torch.tensor([100, 0], dtype=torch.int32, device="cuda")))
    del far
    torch.cuda.empty_cache()


# ------------------------------------------------------------- attention with shaped scores ---

@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_shaped_attention_masked_values_have_no_influence(shape):
    for bad in (math.nan, math.inf, -math.inf):
        for dtype, dim in (("bf16", 128), ("fp16", 72)):
            c = attn_case(14, dtype, 4, 2, dim, [1, 3], [30, 70], 96)
            for b, n in enumerate((30, 70)):
                c["k"][b * 96 + n:(b + 1) * 96] = bad
                c["v"][b * 96 + n:(b + 1) * 96] = bad
            s = shape_of(c, shape)
            check_shaped(c, s)
            c = attn_case(15, dtype, 4, 2, dim, [150])
            s = shape_of(c, shape)
            if s["prefix"] is not None:
                s["prefix"] = torch.tensor([60], dtype=torch.int32)
            clean, clean_lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **on_gpu(s))
            kept = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], clean, clean_lse, **offs(c), **on_gpu(s))
            c["k"][100], c["v"][100] = bad, bad
            out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **on_gpu(s))
            ref, _, far, _ = H.shaped_attention(c, **s)
            R.within(out[:100], ref[:100], far[:100], "out")
            dq, _, _ = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], clean, clean_lse, **offs(c), **on_gpu(s))
            assert dq[:100].isfinite().all()
            R.within(dq[:100], kept[0][:100].double(), kept[0][:100].double().abs() * R.half_step(DT[dtype]) * 2 + 0.05, "dq")


def test_shaped_attention_that_changes_nothing():
    """A prefix of no length, slopes of 0: what attention itself answers."""
    for dtype in ("bf16", "fp16"):
        c = attn_case(70, dtype, 6, 2, 80, [200, 1, 77])
        out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c))
        grads = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c))
        zero = dict(prefix=torch.zeros(3, dtype=torch.int32, device="cuda"))
        a, b = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **zero)
        assert torch.equal(a, out) and torch.equal(b, lse)
        assert all(torch.equal(x, y) for x, y in zip(F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c), **zero), grads))
        for s in (dict(cap=None, slopes=torch.zeros(6), prefix=None), dict(cap=1e4, slopes=None, prefix=None)):
            check_shaped(c, s)                             # (a cap takes digits: some 2^-22 of it, which the bound counts)


def test_shaped_attention_saturated_scores():
    """Scores far beyond the cap: weights of equals, no gradient through them; and scores of infinity."""
    c = attn_case(71, "fp16", 2, 1, 64, [90])
    c["q"].mul_(200.0)
    check_shaped(c, dict(cap=3.0, slopes=None, prefix=None), scale=10.0)
    c["q"][50, 0, 0] = math.inf
    out, _ = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), cap=3.0)
    assert out[:50].isfinite().all() and out[51:].isfinite().all()


def test_shaped_attention_gradient_against_differences():
    """The gradient's direction: along it, the loss of the reference in 64 bits changes as it says."""
    for name in sorted(SHAPES):
        c = attn_case(72, "bf16", 4, 2, 64, [40, 9])
        s = shape_of(c, name)
        out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **on_gpu(s))
        grads = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c), **on_gpu(s))
        big = {n: c[n].double().cpu() for n in "qkv"}

        def loss(step):
            moved = dict(c, **{n: big[n] + step * g.double().cpu() / total for n, g in zip("qkv", grads)})
            return float((H.shaped_attention(dict(moved, q=moved["q"]), **s)[0] * c["dout"].double().cpu()).sum())

        total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
        slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
        # dq, dk and dv are each off by a few half steps of bf16 in the 2-norm: their squares' sum by some 2^-7
        assert abs(slope - total) <= 0.02 * total, (name, slope, total)


def test_shaped_attention_same_results_again():
    c = attn_case(73, "fp16", 8, 2, 128, [300, 77])
    for name in sorted(SHAPES):
        s = on_gpu(shape_of(c, name))
        out, lse = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **s)
        grads = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, **offs(c), **s)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        out2, lse2 = F.fuse_attention(c["q"], c["k"], c["v"], **offs(c), **s, stream=side)
        again = F.fuse_attention_backward(c["dout"], c["q"], c["k"], c["v"], out2, lse2, **offs(c), **s, stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(grads, again))


# ------------------------------------------------------------------------------ all together ---

def serve_state(seed, t=torch.bfloat16):
    """Three sequences that go on by some tokens each."""
    c = cache_case(seed, "bf16" if t == torch.bfloat16 else "fp16", 8, 2, 64, 16, [1, 4, 2], [40, 90, 17])
    g = gen(seed + 1)
    c["qkv"] = rnd(g, (7, 12, 64), t).cuda()
    c["w"] = rnd(g, (64,), t, 0.2, 1.0).cuda()
    c["at"] = torch.tensor([39, 86, 87, 88, 89, 15, 16], dtype=torch.int32).cuda()
    c["freqs"] = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).cuda()
    return c


def serve(c):
    """What a block does with a projection of new tokens: norms and rotation in place, into the cache, attention over it."""
    q, k, v = c["qkv"][:, :8], c["qkv"][:, 8:10], c["qkv"][:, 10:]
    q, k = F.fuse_qk_rotary(q, k, c["at"], c["freqs"], q_weight=c["w"], k_weight=c["w"])
    F.fuse_cache_write(k, v, c["cache"], c["offsets"], c["table"], c["lengths"])
    return [q, k] + list(F.fuse_attention_cache(q, c["cache"], c["offsets"], c["table"], c["lengths"], cap=20.0))


def test_serving_step():
    for t in (torch.bfloat16, torch.float16):
        c = serve_state(80, t)
        q, k, out, lse = serve(c)
        check_rotary(dict(q=c["qkv"][:, :8], k=c["qkv"][:, 8:10], q_weight=c["w"], k_weight=c["w"], positions=c["at"], freqs=c["freqs"], sections=None,
                          pairs="halves"), (q, k))
        c.update(k=k, v=c["qkv"][:, 10:], q=q)
        before = [x.clone() for x in c["cache"]]
        check_write(c)                                     # (again: the same)
        assert all(torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a, b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)
                   for a, b in zip(before, c["cache"]))
        want = H.cache_attention(c, cap=20.0)
        R.within(out, want[0], want[2], "out")
        R.within(lse, want[1], want[3], "lse")
        # against attention over the same keys and values before their rounding to 8 bits: some 2^-4 of a value, averaged over many
        keys = torch.zeros(3 * 90, 2, 64, dtype=t, device="cuda")
        values = torch.zeros_like(keys)
        for s, n in enumerate(c["lengths"].tolist()):
            for g in range(2):
                k8, v8, ks, vs = H.cache_rows(c, s, g, n)
                keys[s * 90:s * 90 + n, g], values[s * 90:s * 90 + n, g] = (k8 * ks[:, None]).to(t).cuda(), (v8 * vs[:, None]).to(t).cuda()
        room = torch.arange(0, 4 * 90, 90, dtype=torch.int32, device="cuda")
        near, _ = F.fuse_attention(q, keys, values, c["offsets"], key_offsets=room, key_lengths=c["lengths"], cap=20.0)
        # keys and values are rounded to t on the way (half a step each: scores of size 20 at most by 20 steps), and the results
        assert float((near - out).double().norm() / out.double().norm()) <= 24 * R.half_step(t)


def train_state(seed):
    g = gen(seed)
    t = torch.bfloat16
    c = dict(qkv=rnd(g, (160, 10, 64), t), qw=rnd(g, (64,), t, 0.2, 1.0), kw=rnd(g, (64,), t, 0.2, 1.0), dout=rnd(g, (160, 6, 64), t),
             at=torch.cat([torch.arange(70), torch.arange(90)]).to(torch.int32), offsets=torch.tensor([0, 70, 160], dtype=torch.int32),
             prefix=torch.tensor([11, 30], dtype=torch.int32), freqs=10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32),
             slopes=2.0 ** -torch.arange(1, 7, dtype=torch.float32))
    return {k: v.cuda() for k, v in c.items()}


def train(c):
    """Queries and keys with norms and rotation, shaped attention, and all gradients."""
    q0, k0, v = c["qkv"][:, :6], c["qkv"][:, 6:8], c["qkv"][:, 8:]
    q, k = F.fuse_qk_rotary(q0, k0, c["at"], c["freqs"], q_weight=c["qw"], k_weight=c["kw"])
    shape = dict(cap=15.0, slopes=c["slopes"], prefix=c["prefix"])
    out, lse = F.fuse_attention(q, k, v, c["offsets"], **shape)
    d = torch.empty_like(c["qkv"])
    F.fuse_attention_backward(c["dout"], q, k, v, out, lse, c["offsets"], dq=d[:, :6], dk=d[:, 6:8], dv=d[:, 8:], **shape)
    got = F.fuse_qk_rotary_backward(d[:, :6], d[:, 6:8], q0, k0, c["at"], c["freqs"], q_weight=c["qw"], k_weight=c["kw"], dq=d[:, :6], dk=d[:, 6:8])
    return [out, lse, d, got.dq_weight, got.dk_weight]


def test_training_step():
    c = train_state(90)
    got = train(c)
    big = {n: c[n].double().cpu().requires_grad_(True) for n in ("qkv", "qw", "kw")}
    angle = H.angles(c["at"], c["freqs"], None)
    q = H.rotary(big["qkv"][:, :6], big["qw"], angle, "halves", 1e-6)
    k = H.rotary(big["qkv"][:, 6:8], big["kw"], angle, "halves", 1e-6)
    outs = []
    for (a, b), first in zip(((0, 70), (70, 160)), (11, 30)):
        i = torch.arange(b - a)
        meet = (i[None] <= i[:, None]) | (i < first)[None]
        rows = []
        for h in range(6):
            x = 15.0 * torch.tanh(0.125 * q[a:b, h] @ k[a:b, h // 3].T / 15.0) - float(c["slopes"][h]) * (i[:, None] - i[None]).abs()
            rows.append(torch.softmax(x.masked_fill(~meet, -math.inf), 1) @ big["qkv"][a:b, 8 + h // 3])
        outs.append(torch.stack(rows, 1))
    out = torch.cat(outs)
    want = [out.detach()] + list(torch.autograd.grad((out * c["dout"].double().cpu()).sum(), [big["qkv"], big["qw"], big["kw"]]))
    for g, w, name in zip([got[0]] + got[2:], want, ("out", "dqkv", "dq_weight", "dk_weight")):
        # some eight roundings to bf16 on the way of every value, each off by at most half a step
        err = float((g.double().cpu() - w).norm() / w.norm())
        assert err <= 8 * 2.0 ** -8, (name, err)


def test_steps_in_two_graphs():
    """Two states of both steps, captured without a warm-up, replayed in turn and at once on two streams, against the eager results."""
    states = [(serve_state(81 + i), train_state(91 + i)) for i in range(2)]
    eager = [[t.clone() for t in serve(s) + train(u)] for s, u in states]
    torch.cuda.synchronize()
    graphs, results = [], []
    for s, u in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(serve(s) + train(u))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for t in results[0] + results[1]:
            t.zero_()
        for s, _ in states:                                # what the replay writes again
            s["cache"].k.view(torch.uint8)[int(s["table"][0, 2]), :, 7] = 0
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
        serve(states[turn % 2][0])                         # the program's own work between the replays
        train(states[turn % 2][1])
        torch.cuda.synchronize()


def test_calls_of_several_threads():
    import threading
    cases = [(serve_state(84 + i), train_state(94 + i)) for i in range(3)]
    want = [[t.clone() for t in serve(s) + train(u)] for s, u in cases]
    torch.cuda.synchronize()
    got, errors = [None] * 3, []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    got[i] = serve(cases[i][0]) + train(cases[i][1])
            stream.synchronize()
        except Exception as e:                             # (looked at below, in the test's own thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
