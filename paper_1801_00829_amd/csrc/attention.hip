// Attention over packed sequences, forward (fuse_attention).
#include "attention.h"

namespace {

using namespace fuse;

constexpr int kRows = 128;                 // rows per tile

// A wave per row.
template <typename T>
__global__ void __launch_bounds__(256) attention_kernel(const AttnArgs a)
{
    const int kvh = blockIdx.x % a.kv_heads;
    const long long t = blockIdx.x / a.kv_heads;
    const int s = seq_of_tile(a, a.q_off, a.q_tokens, a.group, kRows, t);
    const Seq x = seq_at(a, s);
    const long long first = (t - first_tile(x.q0 * a.group, s, kRows)) * kRows, end = min(first + kRows, (long long)x.nq * a.group);
    for (long long r = first + (threadIdx.x >> 6); r < end; r += 4)
        attend_row<T>(a, x, (int)(r / a.group), kvh * a.group + (int)(r % a.group));
}

int attention_impl(const fuse_attn *f, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_attn(f);
    if (rc)
        return rc;
    if ((rc = check_rows(f, out, out_token_ld, out_head_ld, f->heads, f->q_tokens, "out")))
        return rc;
    if (reinterpret_cast<uintptr_t>(lse) % 4)
        return report(FUSE_EINVAL, "lse is not aligned to its type");
    (void)workspace;
    (void)workspace_bytes;
    if (f->q_tokens == 0 || f->seqs == 0)
        return FUSE_OK;
    AttnArgs a = attn_args(f);
    a.out = {out, out_token_ld, out_head_ld};
    a.lse = lse;
    const long long tiles = first_tile(f->q_tokens * a.group, (int)f->seqs, kRows);
    const unsigned blocks = (unsigned)(tiles * f->kv_heads);
    if (f->dtype == FUSE_BF16)
        attention_kernel<__bf16><<<blocks, 256, 0, (hipStream_t)stream>>>(a);
    else
        attention_kernel<_Float16><<<blocks, 256, 0, (hipStream_t)stream>>>(a);
    return launched("attention_kernel");
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
    if (token_ld > (INT64_C(1) << 31) || head_ld > (INT64_C(1) << 40))
        return report(FUSE_EUNSUPPORTED, std::string(what) + ": stride too large");
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
    if (!(f->scale > 0.0) || !(f->scale < 1e30))
        return report(FUSE_EINVAL, "scale must be positive and finite");
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
    return a;
}

}  // namespace fuse

extern "C" {

size_t fuse_attention_bytes(const fuse_attn *attn)
{
    (void)attn;
    return 0;
}

int fuse_attention(const fuse_attn *attn, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return attention_impl(attn, out, out_token_ld, out_head_ld, lse, workspace, workspace_bytes, stream); });
}

}  // extern "C"
