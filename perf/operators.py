"""The calls that a transformer block's operators are measured on: attention over packed sequences, the norms around a
block with its gate and residual scale, and the norm of all gradients with clipping.

Every operator has a plain form (elementary torch operations in 32 bits, rounded once at the end; 64 bits for the sum of
squares over all gradients, which is a 64 bit result) and a definition in 64 bits.  Sizes are generic: token counts from one
to some ten thousand, widths and head layouts of the usual kinds, odd and ragged ones among them.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "fp64": torch.float64}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "fp64": 8}


def listed():
    return [
        # four sequences that generate a token each: the norm after a block's branch, the residual, the norm before the next
        dict(name="norm_token", op="norm", dtype="bf16", rows=4, cols=4096, kind="rms", post=True, gate="none", scale=1.0),
        # the same over the tokens of long prompts, the branch scaled per channel
        dict(name="norm_prompt", op="norm", dtype="bf16", rows=16384, cols=4096, kind="rms", post=True, gate="rowvec", scale=0.5),
        # the same in training: all gradients of one such step
        dict(name="norm_grad", op="norm_grad", dtype="bf16", rows=16384, cols=4096, kind="rms", post=True, gate="rowvec", scale=0.5),
        # a block with layer norms and a gate per cell, rows of odd length, fp32
        dict(name="norm_grad_odd", op="norm_grad", dtype="fp32", rows=5003, cols=1111, kind="layer", post=True, gate="matrix", scale=1.0),
        # one sequence that generates a token, a short history: latency counts
        dict(name="attention_one", op="attention", dtype="fp16", heads=8, kv_heads=1, dim=64, seqs=1, new=1, room=512, spread=1),
        # sixteen sequences that generate a token each, over histories of different length in a cache with room
        dict(name="attention_token", op="attention", dtype="bf16", heads=32, kv_heads=8, dim=128, seqs=16, new=1, room=8192, spread=2),
        # three long prompts of different length, packed
        dict(name="attention_prompt", op="attention", dtype="bf16", heads=32, kv_heads=8, dim=128, seqs=3, new=0, tokens=12288, spread=3),
        # many short prompts of different length, packed; a head of its own for every query head
        dict(name="attention_short", op="attention", dtype="fp16", heads=16, kv_heads=16, dim=64, seqs=61, new=0, tokens=7001, spread=4),
        # training over packed documents: the gradients of queries, keys and values
        dict(name="attention_grad", op="attention_grad", dtype="bf16", heads=32, kv_heads=8, dim=128, seqs=4, new=0, tokens=8192, spread=5),
        # the same with a head size between the usual ones, three query heads to a key head, odd lengths
        dict(name="attention_grad_odd", op="attention_grad", dtype="fp16", heads=12, kv_heads=4, dim=80, seqs=7, new=0, tokens=3331, spread=6),
        # clipping the gradients of a small model in fp64: latency counts
        dict(name="clip_small", op="clip", kinds="fp64", tensors=14, cells=120000, spread=7, clipped=True),
        # clipping the gradients of some layers of a large model, matrices in bf16 and vectors in fp32
        dict(name="clip_layers", op="clip", kinds="bf16+fp32", tensors=54, cells=700000000, spread=8, clipped=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "attention", "attention", "attention_grad", "clip"])
    if op in ("norm", "norm_grad"):
        cols = rng.choice([_log_int(rng, 64, 8192), 8 * _log_int(rng, 16, 1024)])
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), rows=_log_int(rng, 1, 33000000 // cols), cols=cols,
                    kind=rng.choice(["rms", "rms", "layer"]), post=rng.random() < 0.6,
                    gate=rng.choice(["none", "rowvec", "colvec", "matrix"]), scale=rng.choice([1.0, 0.5, 0.1767766952966369]))
    if op == "clip":
        return dict(op=op, kinds=rng.choice(["bf16+fp32", "fp32", "fp16", "fp64", "bf16"]), tensors=rng.randint(1, 60),
                    cells=_log_int(rng, 1000, 300000000), spread=rng.randint(0, 1 << 30), clipped=rng.random() < 0.75)
    kv_heads = rng.choice([1, 2, 4, 8])
    heads, dim = kv_heads * rng.randint(1, 8), rng.choice([64, 128, 8 * rng.randint(4, 16)])
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16"]), heads=heads, kv_heads=kv_heads, dim=dim,
                spread=rng.randint(0, 1 << 30))
    if op == "attention" and rng.random() < 0.4:
        seqs = _log_int(rng, 1, 64)
        return dict(case, seqs=seqs, new=rng.choice([1, 1, 1, rng.randint(2, 16)]), room=_log_int(rng, 64, min(32768, 1000000 // (seqs * kv_heads))))
    tokens = _log_int(rng, 16, 8192 if heads <= 32 else 4096)
    return dict(case, seqs=_log_int(rng, 1, max(1, min(64, tokens // 16))), new=0, tokens=tokens)


# ------------------------------------------------------------------------------------------------ sizes of a case ---

def _shares(case, total):
    """Lengths of the sequences: shares of `total` between one and nine to one; with four sequences and more one has none."""
    r = random.Random(case["spread"])
    w = [r.uniform(0.2, 1.8) for _ in range(case["seqs"])]
    if case["seqs"] >= 4:
        w[case["seqs"] // 2] = 0.0
    lens = [int(total * x / sum(w)) for x in w]
    lens[0] += total - sum(lens)
    return lens


def _lengths(case):
    """(new tokens, tokens that they may look at) of every sequence."""
    if case["new"]:
        r = random.Random(case["spread"])
        return [case["new"]] * case["seqs"], [max(case["new"], int(case["room"] * r.uniform(0.3, 1.0))) for _ in range(case["seqs"])]
    lens = _shares(case, case["tokens"])
    return lens, lens


def _tensors(case):
    """(shape, type) of every gradient: matrices between one and nine to one in size, every sixth one a vector."""
    r = random.Random(case["spread"])
    kinds = case["kinds"].split("+")
    w = [r.uniform(0.2, 1.8) * (0.0005 if i % 6 == 5 else 1.0) for i in range(case["tensors"])]
    found = []
    for i, x in enumerate(w):
        cells = max(1, int(case["cells"] * x / sum(w)))
        vector = i % 6 == 5
        rows = 1 if vector else max(1, int(math.sqrt(cells) * r.uniform(0.5, 2.0)))
        shape = (cells,) if vector else (rows, max(1, cells // rows))
        found.append((shape, kinds[-1] if vector else kinds[0]))
    return found


def work(case):
    if case["op"] in ("norm", "norm_grad"):
        cells, back = case["rows"] * case["cols"], case["op"] == "norm_grad"
        per_cell = (6 if back else 4) + (0 if case["gate"] != "matrix" else 2 if back else 1)
        return {"bytes": per_cell * cells * SIZE[case["dtype"]], "flops": (30 if back else 12) * cells}
    if case["op"] == "clip":
        cells = [(math.prod(shape), SIZE[kind]) for shape, kind in _tensors(case)]
        return {"bytes": sum(2 * c * s for c, s in cells), "flops": sum(3 * c for c, s in cells)}
    new, seen = _lengths(case)
    pairs = sum(n * (s - n) + n * (n + 1) // 2 for n, s in zip(new, seen))
    q, kv = sum(new) * case["heads"] * case["dim"], sum(seen) * case["kv_heads"] * case["dim"]
    if case["op"] == "attention":
        return {"bytes": 2 * (2 * q + 2 * kv) + 4 * sum(new) * case["heads"], "flops": 4 * pairs * case["heads"] * case["dim"]}
    return {"bytes": 2 * (4 * q + 4 * kv) + 4 * sum(new) * case["heads"], "flops": 10 * pairs * case["heads"] * case["dim"]}


# --------------------------------------------------------------------------------------------------------- inputs ---

def _normal(g, shape, dtype, std=1.0, mean=0.0):
    t = torch.empty(shape, dtype=torch.float64 if dtype == "fp64" else torch.float32, device="cuda")
    return t.normal_(mean, std, generator=g).to(DTYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] in ("norm", "norm_grad"):
        return _prepare_norm(case, g)
    if case["op"] == "clip":
        return _prepare_clip(case, g)
    return _prepare_attention(case, g)


def _prepare_norm(case, g):
    rows, cols, t = case["rows"], case["cols"], case["dtype"]
    s = dict(case=case, x=_normal(g, (rows, cols), t, 2.0), z=_normal(g, (rows, cols), t, 0.7, 0.1))
    layer = case["kind"] == "layer"
    for name in ("post", "pre"):
        weight = _normal(g, (cols,), t, 0.2, 1.0)
        s[name] = (weight, _normal(g, (cols,), t, 0.1)) if layer else weight
    if not case["post"]:
        s["post"] = None
    shape = {"none": None, "rowvec": (cols,), "colvec": (rows,), "matrix": (rows, cols)}[case["gate"]]
    s["gate"] = None if shape is None else (case["gate"], _normal(g, shape, t, 0.3, 0.5))
    if case["op"] == "norm_grad":
        s["dh"], s["dy"] = _normal(g, (rows, cols), t, 0.02), _normal(g, (rows, cols), t, 0.02)
        s["h"], s["x"] = s["x"], None                     # the residual stream behind the block, as the forward call left it
    return s


def _prepare_clip(case, g):
    grads = [_normal(g, shape, kind, 0.01) for shape, kind in _tensors(case)]
    total = 0.01 * math.sqrt(sum(t.numel() for t in grads))
    return dict(case=case, grads=grads, out=[torch.empty_like(t) for t in grads], max_norm=(0.3 if case["clipped"] else 30.0) * total)


def _prepare_attention(case, g):
    new, seen = _lengths(case)
    hq, hk, d, t = case["heads"], case["kv_heads"], case["dim"], case["dtype"]
    ends = [0]
    for n in new:
        ends.append(ends[-1] + n)
    s = dict(case=case, scale=1.0 / math.sqrt(d), offsets=torch.tensor(ends, dtype=torch.int32, device="cuda"))
    if case["new"]:                                       # a cache: `room` places for every sequence, `seen` of them in use
        s["q"] = _normal(g, (ends[-1], hq, d), t)
        s["k"], s["v"] = _normal(g, (case["seqs"] * case["room"], hk, d), t), _normal(g, (case["seqs"] * case["room"], hk, d), t)
        s["key_offsets"] = torch.arange(0, (case["seqs"] + 1) * case["room"], case["room"], dtype=torch.int32, device="cuda")
        s["key_lengths"] = torch.tensor(seen, dtype=torch.int32, device="cuda")
    else:                                                 # one projection gives queries, keys and values side by side
        qkv = _normal(g, (ends[-1], hq + 2 * hk, d), t)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["key_offsets"] = s["key_lengths"] = None
    s["longest"] = (max(new), max(seen))
    if case["op"] == "attention_grad":
        s["dout"] = _normal(g, (ends[-1], hq, d), t)
        s["out"], s["lse"] = _attention(s)                # what the forward call returned
    return s


# ----------------------------------------------------------------------------------------------------- plain forms ---

def _norm_of(v, weight, kind, eps=1e-6):
    """(normalised v, what it was multiplied with, weighted result)"""
    w, b = weight if isinstance(weight, tuple) else (weight, None)
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + eps)
    n = v * r
    y = n * w.float()
    return n, r, y if b is None else y + b.float()


def _gate_of(gate):
    if gate is None:
        return None
    kind, t = gate
    return t.float()[:, None] if kind == "colvec" else t.float()


def _norm(s):
    kind, t = s["case"]["kind"], s["x"].dtype
    u = s["z"].float()
    if s["post"] is not None:
        u = _norm_of(u, s["post"], kind)[2]
    gate = _gate_of(s["gate"])
    if gate is not None:
        u = u * gate
    h = s["x"].float() + s["case"]["scale"] * u
    return {"h": h.to(t), "y": _norm_of(h, s["pre"], kind)[2].to(t)}


def _norm_back(dy, n, r, weight, kind):
    """Gradient of a norm's input, weight and bias."""
    w, b = weight if isinstance(weight, tuple) else (weight, None)
    g = dy * w.float()
    d = r * (g - n * (g * n).mean(1, keepdim=True))
    if kind == "layer":
        d = d - r * g.mean(1, keepdim=True)
    return d, (dy * n).sum(0), None if b is None else dy.sum(0)


def _norm_grad(s):
    kind, t, scale = s["case"]["kind"], s["h"].dtype, s["case"]["scale"]
    n, r, _ = _norm_of(s["h"].float(), s["pre"], kind)
    d, dpre, dpre_bias = _norm_back(s["dy"].float(), n, r, s["pre"], kind)
    dx = s["dh"].float() + d
    out = {"dx": dx, "dpre": dpre, "dpre_bias": dpre_bias}
    u, du, gate = s["z"].float(), scale * dx, _gate_of(s["gate"])
    if s["post"] is not None:
        n, r, u = _norm_of(u, s["post"], kind)
    if gate is not None:
        dgate = du * u
        out["dgate"] = {"rowvec": lambda: dgate.sum(0), "colvec": lambda: dgate.sum(1), "matrix": lambda: dgate}[s["gate"][0]]()
        du = du * gate
    if s["post"] is not None:
        du, out["dpost"], out["dpost_bias"] = _norm_back(du, n, r, s["post"], kind)
    out["dz"] = du
    return {k: v.to(t) for k, v in out.items() if v is not None}


def _padded(s):
    """Queries (sequences, key heads, query heads of one * longest, dim), keys and values (sequences, key heads, longest,
    dim), which pairs may meet, and the places of the queries and keys in the packed tensors."""
    q, k, v, hk = s["q"], s["k"], s["v"], s["case"]["kv_heads"]
    lq, lk = s["longest"]
    starts, ends = s["offsets"][:-1].long(), s["offsets"][1:].long()
    n = ends - starts
    first, seen = (starts, n) if s["key_offsets"] is None else (s["key_offsets"][:-1].long(), s["key_lengths"].long())
    i, j = torch.arange(lq, device=q.device), torch.arange(lk, device=q.device)
    at_q = torch.where(i < n[:, None], starts[:, None] + i, q.shape[0])
    at_k = torch.where(j < seen[:, None], first[:, None] + j, k.shape[0])
    meet = (j <= (i + (seen - n)[:, None])[:, :, None]) & (i < n[:, None])[:, :, None] & (j < seen[:, None])[:, None, :]
    return _rows(q, at_q, hk), _rows(k, at_k, hk), _rows(v, at_k, hk), meet, at_q, at_k


def _rows(x, at, hk):
    """Packed (tokens, heads, dim) -> (sequences, key heads, heads of one * longest, dim) in 32 bits, 0 behind a sequence's end."""
    x = torch.cat([x.float(), x.new_zeros((1,) + x.shape[1:], dtype=torch.float32)])[at]
    b, l, h, d = x.shape
    return x.view(b, l, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, (h // hk) * l, d)


def _packed(x, at, tokens, longest):
    """The way back of _rows."""
    b, hk, gl, d = x.shape
    x = x.view(b, hk, gl // longest, longest, d).permute(0, 3, 1, 2, 4).reshape(b, longest, -1, d)
    out = torch.zeros((tokens + 1,) + x.shape[2:], dtype=x.dtype, device=x.device)
    out[at] = x
    return out[:tokens]


def _scores(s, q, k, meet):
    x = torch.matmul(q, k.transpose(-1, -2).contiguous())
    b, hk, gl, lk = x.shape
    x.view(b, hk, -1, meet.shape[1], lk).mul_(s["scale"]).masked_fill_(~meet[:, None, None], -math.inf)
    return x


def _attention(s):
    q, k, v, meet, at_q, _ = _padded(s)
    x = _scores(s, q, k, meet)
    top = x.amax(-1, keepdim=True).clamp_min_(torch.finfo(torch.float32).min)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.clamp_min(1e-30)
    lse = top + total.log()
    tokens, lq = s["q"].shape[0], s["longest"][0]
    return _packed(out, at_q, tokens, lq).to(s["q"].dtype), _packed(lse, at_q, tokens, lq)[..., 0].contiguous()


def _attention_grad(s):
    q, k, v, meet, at_q, at_k = _padded(s)
    hk, tokens, (lq, lk) = s["case"]["kv_heads"], s["q"].shape[0], s["longest"]
    dout = _rows(s["dout"], at_q, hk)
    delta = (dout * _rows(s["out"], at_q, hk)).sum(-1, keepdim=True)
    p = _scores(s, q, k, meet).sub_(_rows(s["lse"][..., None], at_q, hk)).exp_()
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), dout)
    ds = torch.matmul(dout, v.transpose(-1, -2).contiguous()).sub_(delta).mul_(p).mul_(s["scale"])
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q)
    t = s["q"].dtype
    return {"dq": _packed(dq, at_q, tokens, lq).to(t), "dk": _packed(dk, at_k, s["k"].shape[0], lk).to(t),
            "dv": _packed(dv, at_k, s["k"].shape[0], lk).to(t)}


def _clip(s):
    norm = torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    scaled = [(t * factor if t.dtype == torch.float64 else t.float() * factor.float()).to(t.dtype) for t in s["grads"]]
    return {"norm": norm, "grads": scaled}


# ------------------------------------------------------------------------------------------------ the library's calls ---

def _own(s):
    import paper_1801_00829_amd as F
    case = s["case"]
    if case["op"] == "norm":
        h, y = F.fuse_block_norm(s["x"], s["z"], gate=s["gate"], scale=case["scale"], post=s["post"], pre=s["pre"], kind=case["kind"])
        return {"h": h, "y": y}
    if case["op"] == "norm_grad":
        got = F.fuse_block_norm_backward(s["dh"], s["dy"], s["h"], s["z"], gate=s["gate"], scale=case["scale"], post=s["post"],
                                         pre=s["pre"], kind=case["kind"])
        return {k: v for k, v in got._asdict().items() if v is not None}
    if case["op"] == "clip":
        norm = F.fuse_grad_clip(s["grads"], s["max_norm"], out=s["out"])
        return {"norm": norm.view(()), "grads": s["out"]}
    if case["op"] == "attention":
        return F.fuse_attention(s["q"], s["k"], s["v"], s["offsets"], key_offsets=s["key_offsets"], key_lengths=s["key_lengths"],
                                scale=s["scale"])
    dq, dk, dv = F.fuse_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["offsets"], scale=s["scale"])
    return {"dq": dq, "dk": dk, "dv": dv}


def run(state):
    if own:
        return _own(state)
    return {"norm": _norm, "norm_grad": _norm_grad, "clip": _clip, "attention": _attention,
            "attention_grad": _attention_grad}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------- definitions in 64 bits ---

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        big = [t.to(torch.float64) for t in s["grads"]]
        norm = math.sqrt(sum(float(torch.dot(t.flatten(), t.flatten())) for t in big))
        factor = min(1.0, s["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": [t.mul_(factor) for t in big]}
    return _exact_norm(case, s) if case["op"] in ("norm", "norm_grad") else _exact_attention(case, s)


def _exact_norm(case, s):
    """By automatic differentiation in 64 bits."""
    def big(t):
        return None if t is None else t.detach().double().requires_grad_(True)

    def norm(v, w, b):
        if case["kind"] == "layer":
            c = v - v.sum(1, keepdim=True) / v.shape[1]
            return c / ((c * c).sum(1, keepdim=True) / v.shape[1] + 1e-6).sqrt() * w + b
        return v / ((v * v).sum(1, keepdim=True) / v.shape[1] + 1e-6).sqrt() * w

    def both(p):
        return (None, None) if p is None else (big(p[0]), big(p[1])) if isinstance(p, tuple) else (big(p), None)

    post, pre, z, gate = both(s["post"]), both(s["pre"]), big(s["z"]), big(s["gate"][1]) if s["gate"] else None
    u = z if post[0] is None else norm(z, *post)
    if gate is not None:
        u = u * (gate.unsqueeze(1) if case["gate"] == "colvec" else gate)
    if case["op"] == "norm":
        with torch.no_grad():
            h = s["x"].double() + case["scale"] * u
            return {"h": h, "y": norm(h, *pre)}
    h = big(s["h"])
    dh, dpre, *dpre_bias = torch.autograd.grad(norm(h, *pre), [t for t in (h,) + pre if t is not None], s["dy"].double())
    out = {"dx": s["dh"].double() + dh, "dpre": dpre}
    if dpre_bias:
        out["dpre_bias"] = dpre_bias[0]
    leaves = {k: t for k, t in (("dz", z), ("dgate", gate), ("dpost", post[0]), ("dpost_bias", post[1])) if t is not None}
    out.update(zip(leaves, torch.autograd.grad(u, list(leaves.values()), case["scale"] * out["dx"])))
    return out


def _exact_attention(case, s):
    """Sequence by sequence and head by head in 64 bits."""
    new, seen = _lengths(case)
    group = case["heads"] // case["kv_heads"]
    back = case["op"] == "attention_grad"
    q = s["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    dk = torch.zeros(s["k"].shape, dtype=torch.float64, device=q.device)
    dv = torch.zeros_like(dk)
    at = 0
    for b, (n, m) in enumerate(zip(new, seen)):
        first = b * case["room"] if case["new"] else at
        later = torch.arange(m, device=q.device)[None, :] > torch.arange(n, device=q.device)[:, None] + (m - n)
        for h in range(case["heads"] if n else 0):
            qh, kh, vh = q[at:at + n, h].double(), s["k"][first:first + m, h // group].double(), s["v"][first:first + m, h // group].double()
            x = (qh @ kh.T * s["scale"]).masked_fill(later, -math.inf)
            if not back:
                lse[at:at + n, h] = torch.logsumexp(x, 1)
                out[at:at + n, h] = torch.softmax(x, 1) @ vh
                continue
            g = s["dout"][at:at + n, h].double()
            p = torch.exp(x - s["lse"][at:at + n, h].double()[:, None])
            dx = p * (g @ vh.T - (g * s["out"][at:at + n, h].double()).sum(1)[:, None]) * s["scale"]
            out[at:at + n, h] = dx @ kh
            dk[first:first + m, h // group] += dx.T @ qh
            dv[first:first + m, h // group] += p.T @ g
        at += n
    return {"dq": out, "dk": dk, "dv": dv} if back else (out, lse)
