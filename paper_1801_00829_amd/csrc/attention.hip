// Attention over packed sequences, forward: checks, launch shapes and C entry points (kernels: attention_forward.h).
#include "attention_forward.h"

namespace fuse {
namespace forward {
#define FUSE_SHAPES(T) FUSE_FORWARD(extern, T, 1) FUSE_FORWARD(extern, T, 3) FUSE_FORWARD(extern, T, 5) FUSE_FORWARD(extern, T, 7)
FUSE_SHAPES(__bf16)
FUSE_SHAPES(_Float16)
}  // namespace forward
}  // namespace fuse

namespace {

using namespace fuse;
using namespace fuse::forward;

long long tiles_of(const fuse_attn *f) { return first_tile(f->q_tokens * (f->heads / f->kv_heads), (int)f->seqs, kRows); }

// Splits of the keys: as many as it takes to have two blocks for each of 256 compute units, of at least four steps each where all
// sequences are equally long (two: of at least eight): a step takes about a microsecond alone, the launch that joins them seven.  One token
// of 32 heads over 8, dim 128, over 32768 places: 33 us with 64 splits; two tokens over 1500 places each: 17 us with splits of four steps,
// 23 with splits of eight; 8 heads over 1, dim 64, over 512 places: 12 us without a split, 19 with two.  The lengths are the device's: a long
// history among many short ones, or one that fills little of its room, has the splits of the mean room.
int splits_of(const fuse_attn *f)
{
    const long long blocks = tiles_of(f) * f->kv_heads, keys = f->k_tokens / (f->seqs > 0 ? f->seqs : 1);
    long long n = blocks > 0 ? 512 / blocks : 1;
    n = n < keys / (4 * kKeys) ? n : keys / (4 * kKeys);
    if (n == 2 && keys < 16 * kKeys)
        n = 1;
    return (int)(n < 1 ? 1 : n > kMaxSplits ? kMaxSplits : n);
}

size_t parts_floats(const fuse_attn *f, int splits)
{
    return splits > 1 ? (size_t)f->q_tokens * f->heads * splits * (f->dim + 2) : 0;
}

template <typename T>
int launch_shape(int shape, const AttnArgs &a, const Parts &p, unsigned tiles, hipStream_t s)
{
    switch (shape) {
    case kPlain: return launch<T, kPlain>(a, p, tiles, s);
    case kShaped: return launch<T, kShaped>(a, p, tiles, s);
    case kShaped | kCapped: return launch<T, kShaped | kCapped>(a, p, tiles, s);
    case kShaped | kSloped: return launch<T, kShaped | kSloped>(a, p, tiles, s);
    default: return launch<T, kShaped | kCapped | kSloped>(a, p, tiles, s);
    }
}

int attention_impl(const fuse_attn *f, const fuse_attn_shape *shape, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_attn(f);
    if (rc || (rc = check_shape(f, shape)))
        return rc;
    if ((rc = check_rows(f, out, out_token_ld, out_head_ld, f->heads, f->q_tokens, "out")))
        return rc;
    if (reinterpret_cast<uintptr_t>(lse) % 4)
        return report(FUSE_EINVAL, "lse is not aligned to its type");
    if (f->q_tokens == 0 || f->seqs == 0)
        return FUSE_OK;
    AttnArgs a = attn_args(f);
    a.out = {out, out_token_ld, out_head_ld};
    a.lse = lse;
    set_shape(a, shape);
    Parts p = {};
    p.splits = splits_of(f);
    const size_t need = parts_floats(f, p.splits) * sizeof(float);
    if (need && (!workspace || !on_16_bytes(workspace) || workspace_bytes < need))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(need) + " bytes on 16 are needed");
    p.o = static_cast<float *>(workspace);
    p.m = p.o + (size_t)f->q_tokens * f->heads * p.splits * f->dim;
    p.l = p.m + (size_t)f->q_tokens * f->heads * p.splits;
    const unsigned tiles = (unsigned)tiles_of(f);
    return f->dtype == FUSE_BF16 ? launch_shape<__bf16>(shape_of(shape), a, p, tiles, (hipStream_t)stream)
                                 : launch_shape<_Float16>(shape_of(shape), a, p, tiles, (hipStream_t)stream);
}

}  // namespace

namespace fuse {

int check_rows(const fuse_attn *f, const void *p, int64_t token_ld, int64_t head_ld, int64_t heads, int64_t tokens, const char *what)
{
    if (!p)
        return tokens > 0 && f->seqs > 0 ? report(FUSE_EINVAL, std::string(what) + " is NULL") : FUSE_OK;
    if (!on_16_bytes(p) || token_ld % 8 || head_ld % 8)
        return report(FUSE_EUNSUPPORTED, std::string(what) + ": rows are not on 16 bytes");
    if ((tokens > 1 && token_ld < f->dim) || (heads > 1 && head_ld < f->dim))
        return report(FUSE_ESHAPE, std::string(what) + ": stride < dim");
    if (token_ld > (INT64_C(1) << 40) || head_ld > (INT64_C(1) << 40))
        return report(FUSE_EUNSUPPORTED, std::string(what) + ": stride > 2^40");
    return FUSE_OK;
}

int check_attn(const fuse_attn *f)
{
    if (!f)
        return report(FUSE_EINVAL, "attn is NULL");
    if (!known_dtype(f->dtype))
        return report(FUSE_EINVAL, "dtype is not a fuse_dtype");
    if (f->heads < 1 || f->kv_heads < 1 || f->dim < 1 || f->q_tokens < 0 || f->k_tokens < 0 || f->seqs < 0)
        return report(FUSE_EINVAL, "heads, kv_heads and dim must be positive, counts must not be negative");
    if (f->heads % f->kv_heads)
        return report(FUSE_ESHAPE, "heads is no multiple of kv_heads");
    if (!(f->scale >= 1e-30) || !(f->scale <= 1e30))        // (a normal fp32 number: a masked score times it has to stay -inf)
        return report(FUSE_EINVAL, "scale must lie between 1e-30 and 1e30");
    if (f->dtype != FUSE_BF16 && f->dtype != FUSE_F16)
        return report(FUSE_EUNSUPPORTED, "attention takes FUSE_BF16 and FUSE_F16");
    if (f->dim % 8 || f->dim > kMaxDim)
        return report(FUSE_EUNSUPPORTED, "dim is no multiple of 8 up to " + std::to_string(kMaxDim));
    if (f->q_tokens >= (INT64_C(1) << 31) || f->k_tokens >= (INT64_C(1) << 31) || f->seqs >= (1 << 24) || f->heads > 4096 ||
        f->q_tokens * f->heads >= (INT64_C(1) << 36))
        return report(FUSE_EUNSUPPORTED, "2^31 tokens, 2^24 sequences, 4096 heads or 2^36 queries of all heads, or more");
    if ((first_tile(f->q_tokens * (f->heads / f->kv_heads), (int)f->seqs, 32) + first_tile(f->k_tokens, (int)f->seqs, 32)) * f->kv_heads >= (1 << 24))
        return report(FUSE_EUNSUPPORTED, "more tiles of queries or keys than one launch has blocks");
    if (f->seqs > 0 && !f->q_offsets)
        return report(FUSE_EINVAL, "q_offsets is NULL");
    if (f->seqs > 0 && !f->k_offsets && f->k_tokens != f->q_tokens)
        return report(FUSE_ESHAPE, "without k_offsets, k has as many tokens as q");
    const uintptr_t width = f->offsets_are_64 ? 8 : 4;
    for (const void *p : {f->q_offsets, f->k_offsets, f->k_lengths})
        if (reinterpret_cast<uintptr_t>(p) % width)
            return report(FUSE_EINVAL, "offsets or lengths are not aligned to their type");
    int rc = check_rows(f, f->q, f->q_token_ld, f->q_head_ld, f->heads, f->q_tokens, "q");
    if (!rc)
        rc = check_rows(f, f->k, f->k_token_ld, f->k_head_ld, f->kv_heads, f->k_tokens, "k");
    if (!rc)
        rc = check_rows(f, f->v, f->v_token_ld, f->v_head_ld, f->kv_heads, f->k_tokens, "v");
    return rc;
}

int check_shape(const fuse_attn *f, const fuse_attn_shape *shape)
{
    if (!shape)
        return FUSE_OK;
    if (shape->cap != 0.0 && (!(shape->cap >= 1e-3) || !(shape->cap <= 1e4)))
        return report(FUSE_EINVAL, "cap must be 0 (none) or lie between 1e-3 and 1e4 (capped scores are off by some 2^-22 of it)");
    if (reinterpret_cast<uintptr_t>(shape->slopes) % 4 || reinterpret_cast<uintptr_t>(shape->prefix_lengths) % (f->offsets_are_64 ? 8 : 4))
        return report(FUSE_EINVAL, "slopes or prefix_lengths are not aligned to their type");
    if (shape->prefix_lengths && !f->causal)
        return report(FUSE_EINVAL, "prefix_lengths goes with causal: without it all queries see all keys");
    return FUSE_OK;
}

int shape_of(const fuse_attn_shape *shape)
{
    if (!shape || (shape->cap == 0.0 && !shape->slopes && !shape->prefix_lengths))
        return kPlain;
    return kShaped | (shape->cap != 0.0 ? kCapped : 0) | (shape->slopes ? kSloped : 0);
}

void set_shape(AttnArgs &a, const fuse_attn_shape *shape)
{
    if (shape)
        a.cap = (float)shape->cap, a.slopes = shape->slopes, a.prefix = shape->prefix_lengths;
}

AttnArgs attn_args(const fuse_attn *f)
{
    AttnArgs a = {};
    a.q = {const_cast<void *>(f->q), f->q_token_ld, f->q_head_ld};
    a.k = {const_cast<void *>(f->k), f->k_token_ld, f->k_head_ld};
    a.v = {const_cast<void *>(f->v), f->v_token_ld, f->v_head_ld};
    a.q_off = f->q_offsets, a.k_off = f->k_offsets ? f->k_offsets : f->q_offsets, a.k_len = f->k_lengths;
    a.q_tokens = f->q_tokens, a.k_tokens = f->k_tokens;
    a.seqs = (int)f->seqs, a.heads = f->heads, a.kv_heads = f->kv_heads, a.group = f->heads / f->kv_heads, a.dim = f->dim;
    a.causal = f->causal != 0, a.off64 = f->offsets_are_64 != 0;
    a.scale = (float)f->scale;
    int n = 0;
    while ((1 << n) < a.group)
        ++n;
    a.div_mul = (unsigned)(((unsigned long long)1 << (31 + n)) / (unsigned)a.group + 1);
    a.div_shift = n > 0 ? n - 1 : 0;
    return a;
}

}  // namespace fuse

extern "C" {

size_t fuse_attention_bytes(const fuse_attn *attn)
{
    return fuse::guard_bytes([&] { return fuse::check_attn(attn) ? 0 : parts_floats(attn, splits_of(attn)) * sizeof(float); });
}

int fuse_attention(const fuse_attn *attn, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return attention_impl(attn, nullptr, out, out_token_ld, out_head_ld, lse, workspace, workspace_bytes, stream); });
}

int fuse_attention_shaped(const fuse_attn *attn, const fuse_attn_shape *shape, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return attention_impl(attn, shape, out, out_token_ld, out_head_ld, lse, workspace, workspace_bytes, stream); });
}

}  // extern "C"
