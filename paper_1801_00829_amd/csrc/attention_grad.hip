// Attention over packed sequences, gradients (fuse_attention_backward).
#include "attention.h"

namespace {

using namespace fuse;

constexpr int kRows = 128;                 // rows, or keys, per tile

// A wave per row; leaves delta for the keys' kernel.
template <typename T>
__global__ void __launch_bounds__(256) attention_query_grad_kernel(const AttnArgs a)
{
    const int kvh = blockIdx.x % a.kv_heads;
    const long long t = blockIdx.x / a.kv_heads;
    const int s = seq_of_tile(a, a.q_off, a.q_tokens, a.group, kRows, t);
    const Seq x = seq_at(a, s);
    const long long first = (t - first_tile(x.q0 * a.group, s, kRows)) * kRows, end = min(first + kRows, (long long)x.nq * a.group);
    for (long long r = first + (threadIdx.x >> 6); r < end; r += 4)
        query_grad_row<T>(a, x, (int)(r / a.group), kvh * a.group + (int)(r % a.group));
}

// A wave per key.
template <typename T>
__global__ void __launch_bounds__(256) attention_key_grad_kernel(const AttnArgs a)
{
    const int kvh = blockIdx.x % a.kv_heads;
    const long long t = blockIdx.x / a.kv_heads;
    const int s = seq_of_tile(a, a.k_off, a.k_tokens, 1, kRows, t);
    const Seq x = seq_at(a, s);
    const long long first = (t - first_tile(x.k0, s, kRows)) * kRows, end = min(first + kRows, (long long)x.nk);
    for (long long j = first + (threadIdx.x >> 6); j < end; j += 4)
        key_grad_row<T>(a, x, (int)j, kvh);
}

size_t backward_bytes(const fuse_attn *f) { return (size_t)f->q_tokens * f->heads * sizeof(float); }

template <typename T>
int launch_grads(const AttnArgs &a, hipStream_t s)
{
    const long long q_tiles = first_tile(a.q_tokens * a.group, a.seqs, kRows), k_tiles = first_tile(a.k_tokens, a.seqs, kRows);
    if (a.q_tokens > 0) {
        attention_query_grad_kernel<T><<<(unsigned)(q_tiles * a.kv_heads), 256, 0, s>>>(a);
        if (const int rc = launched("attention_query_grad_kernel"))
            return rc;
    }
    if (a.k_tokens > 0)
        attention_key_grad_kernel<T><<<(unsigned)(k_tiles * a.kv_heads), 256, 0, s>>>(a);
    return launched("attention_key_grad_kernel");
}

int backward_impl(const fuse_attn *f, const fuse_attn_grads *g, void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_attn(f);
    if (rc)
        return rc;
    if (!g)
        return report(FUSE_EINVAL, "grads is NULL");
    if ((rc = check_rows(f, g->dout, g->dout_token_ld, g->dout_head_ld, f->heads, f->q_tokens, "dout")) ||
        (rc = check_rows(f, g->out, g->out_token_ld, g->out_head_ld, f->heads, f->q_tokens, "out")) ||
        (rc = check_rows(f, g->dq, g->dq_token_ld, g->dq_head_ld, f->heads, f->q_tokens, "dq")) ||
        (rc = check_rows(f, g->dk, g->dk_token_ld, g->dk_head_ld, f->kv_heads, f->k_tokens, "dk")) ||
        (rc = check_rows(f, g->dv, g->dv_token_ld, g->dv_head_ld, f->kv_heads, f->k_tokens, "dv")))
        return rc;
    if (f->seqs == 0 || (f->q_tokens == 0 && f->k_tokens == 0))
        return FUSE_OK;
    if ((!g->lse && f->q_tokens > 0) || reinterpret_cast<uintptr_t>(g->lse) % 4)
        return report(FUSE_EINVAL, "lse is NULL or not aligned to its type");
    if (f->q_tokens > 0 && (!workspace || !on_16_bytes(workspace) || workspace_bytes < backward_bytes(f)))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(backward_bytes(f)) + " bytes on 16 are needed");
    AttnArgs a = attn_args(f);
    a.dout = {const_cast<void *>(g->dout), g->dout_token_ld, g->dout_head_ld};
    a.out = {const_cast<void *>(g->out), g->out_token_ld, g->out_head_ld};
    a.dq = {g->dq, g->dq_token_ld, g->dq_head_ld};
    a.dk = {g->dk, g->dk_token_ld, g->dk_head_ld};
    a.dv = {g->dv, g->dv_token_ld, g->dv_head_ld};
    a.lse = const_cast<float *>(g->lse);
    a.delta = static_cast<float *>(workspace);
    return f->dtype == FUSE_BF16 ? launch_grads<__bf16>(a, (hipStream_t)stream) : launch_grads<_Float16>(a, (hipStream_t)stream);
}

}  // namespace

extern "C" {

size_t fuse_attention_backward_bytes(const fuse_attn *attn)
{
    return attn && attn->q_tokens > 0 && attn->heads > 0 ? backward_bytes(attn) : 0;
}

int fuse_attention_backward(const fuse_attn *attn, const fuse_attn_grads *grads, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return backward_impl(attn, grads, workspace, workspace_bytes, stream); });
}

}  // extern "C"
