// Attention over packed sequences, gradients: checks, launch shapes and C entry points (kernels: attention_backward.h).
#include "attention_backward.h"

namespace fuse {
namespace backward {
#define FUSE_SHAPES(T) FUSE_BACKWARD(extern, T, 1) FUSE_BACKWARD(extern, T, 3) FUSE_BACKWARD(extern, T, 5) FUSE_BACKWARD(extern, T, 7)
FUSE_SHAPES(__bf16)
FUSE_SHAPES(_Float16)
}  // namespace backward
}  // namespace fuse

namespace {

using namespace fuse;
using namespace fuse::backward;

// Zeros in the rows of no sequence, in those of dq, dk and dv that are given: block x takes the rows between two sequences (before the first
// one, behind the last one), y some of them, z = 0 those of the queries, z = 1 those of the keys.  3 to 4 us where there are none.
__global__ void __launch_bounds__(256) attention_rest_kernel(const AttnArgs a)
{
    constexpr int kTokens = 16;            // at a time
    const bool keys = blockIdx.z == 1;
    if (keys ? !a.dk.p && !a.dv.p : !a.dq.p)
        return;
    const int heads = keys ? a.kv_heads : a.heads, chunks = a.dim / 8, per = heads * chunks;
    for (int s = blockIdx.x; s <= a.seqs; s += gridDim.x) {
        long long begin = 0, end = keys ? a.k_tokens : a.q_tokens;
        if (s > 0) {
            const Seq x = seq_at(a, s - 1);
            begin = keys ? x.k0 + x.nk : x.q0 + x.nq;
        }
        if (s < a.seqs) {
            const Seq x = seq_at(a, s);
            end = keys ? x.k0 : x.q0;
        }
        for (long long t = begin + blockIdx.y * kTokens; t < end; t += gridDim.y * kTokens)
            for (int i = threadIdx.x; i < per * kTokens; i += 256) {
                const long long token = t + i / per;
                const int head = i % per / chunks, d = i % chunks * 8;
                if (token >= end)
                    break;
                if (!keys)
                    *reinterpret_cast<uint4 *>(row_of<short>(a.dq, token, head) + d) = make_uint4(0, 0, 0, 0);
                if (keys && a.dk.p)
                    *reinterpret_cast<uint4 *>(row_of<short>(a.dk, token, head) + d) = make_uint4(0, 0, 0, 0);
                if (keys && a.dv.p)
                    *reinterpret_cast<uint4 *>(row_of<short>(a.dv, token, head) + d) = make_uint4(0, 0, 0, 0);
            }
    }
}

// Splits of the rows in the keys' kernel: as many as it takes to have five blocks for each of 256 compute units (two run at a time, and
// they are not equally long), of at least three steps each where all sequences are equally long and half of the pairs are masked.  Whole
// backward passes, without splits and with them: 2048 tokens, 32 heads over 1, dim 128: 1639 and 200 us; two sequences of 2048, 32 over 4: 499 and
// 308 us (with 512 blocks for a goal 499, with 1536 313); 4000 tokens, 32 over 8: 255 and 227 us; 256 tokens, 8 over 8: 22 us either way.
// With a prefix there may be no masked pairs: up to half as many blocks, of three steps of all rows.  Without and with this: 308 tokens of a sequence
// under a prefix, 6 heads over 2, dim 128, 55 and 45 us; 2353 in 16 sequences, 8 over 1, 62 and 53; 5863 in seven, 3 over 1, whose blocks are enough
// already, 131 (148 with such steps up to the whole goal).
int key_splits(const fuse_attn *f, const fuse_attn_shape *shape)
{
    if (f->seqs == 0)
        return 1;
    const long long blocks = first_tile(f->k_tokens, (int)f->seqs, kKeys) * f->kv_heads;
    const long long steps = f->q_tokens * (f->heads / f->kv_heads) / f->seqs / kStep;
    long long n = std::min(1280 / blocks, steps / 2 / 3);
    if (shape && shape->prefix_lengths)
        n = std::max(n, std::min(640 / blocks, steps / 3));
    return (int)(n < 1 ? 1 : n > 32 ? 32 : n);
}

// delta and lse2 (and with slopes every row's place and slope), each with room for a last step's rows behind the last row, and the splits' sums
size_t stat_floats(const fuse_attn *f) { return ((size_t)f->q_tokens * f->heads + kStep + 3) / 4 * 4; }
// (fp16) the lifts
size_t lift_ints(const fuse_attn *f)
{
    return f->dtype == FUSE_F16 ? ((size_t)first_tile(f->q_tokens * (f->heads / f->kv_heads), (int)f->seqs, 32) * f->kv_heads + 3) / 4 * 4 : 0;
}
size_t backward_bytes(const fuse_attn *f, const fuse_attn_shape *shape)
{
    const int splits = key_splits(f, shape);
    return (stat_floats(f) * (shape_of(shape) & kSloped ? 4 : 2) + lift_ints(f) + (splits > 1 ? (size_t)f->k_tokens * f->kv_heads * splits * 2 * f->dim : 0)) * sizeof(float);
}

// The arguments of both calls: the inputs and the results.
AttnArgs grad_args(const fuse_attn *f, const fuse_attn_grads *g)
{
    AttnArgs a = attn_args(f);
    a.dq = {g->dq, g->dq_token_ld, g->dq_head_ld};
    a.dk = {g->dk, g->dk_token_ld, g->dk_head_ld};
    a.dv = {g->dv, g->dv_token_ld, g->dv_head_ld};
    return a;
}

int zero_rest_impl(const fuse_attn *f, const fuse_attn_grads *g, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_attn(f);
    if (rc)
        return rc;
    if (!g)
        return report(FUSE_EINVAL, "grads is NULL");
    if ((g->dq && (rc = check_rows(f, g->dq, g->dq_token_ld, g->dq_head_ld, f->heads, f->q_tokens, "dq"))) ||
        (g->dk && (rc = check_rows(f, g->dk, g->dk_token_ld, g->dk_head_ld, f->kv_heads, f->k_tokens, "dk"))) ||
        (g->dv && (rc = check_rows(f, g->dv, g->dv_token_ld, g->dv_head_ld, f->kv_heads, f->k_tokens, "dv"))))
        return rc;
    if ((!g->dq || f->q_tokens == 0) && ((!g->dk && !g->dv) || f->k_tokens == 0))
        return FUSE_OK;
    const AttnArgs a = grad_args(f, g);
    const unsigned gaps = std::min(a.seqs + 1, 512);
    attention_rest_kernel<<<dim3(gaps, 512 / gaps, 2), 256, 0, (hipStream_t)stream>>>(a);
    return launched("attention_rest_kernel");
}

template <typename T>
int launch_shape(int shape, const AttnArgs &a, hipStream_t s)
{
    switch (shape) {
    case kPlain: return launch_grads<T, kPlain>(a, s);
    case kShaped: return launch_grads<T, kShaped>(a, s);
    case kShaped | kCapped: return launch_grads<T, kShaped | kCapped>(a, s);
    case kShaped | kSloped: return launch_grads<T, kShaped | kSloped>(a, s);
    default: return launch_grads<T, kShaped | kCapped | kSloped>(a, s);
    }
}

int backward_impl(const fuse_attn *f, const fuse_attn_shape *shape, const fuse_attn_grads *g, void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_attn(f);
    if (rc || (rc = check_shape(f, shape)))
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
    if (f->q_tokens > 0 && (!workspace || !on_16_bytes(workspace) || workspace_bytes < backward_bytes(f, shape)))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(backward_bytes(f, shape)) + " bytes on 16 are needed");
    AttnArgs a = grad_args(f, g);
    a.dout = {const_cast<void *>(g->dout), g->dout_token_ld, g->dout_head_ld};
    a.out = {const_cast<void *>(g->out), g->out_token_ld, g->out_head_ld};
    a.lse = const_cast<float *>(g->lse);
    a.delta = static_cast<float *>(workspace);
    a.lse2 = a.delta + stat_floats(f);
    a.lifts = reinterpret_cast<int *>(a.lse2 + stat_floats(f));
    a.parts = a.lse2 + stat_floats(f) + lift_ints(f);
    set_shape(a, shape);
    if (shape_of(shape) & kSloped) {
        a.row_place = reinterpret_cast<int *>(a.parts);
        a.row_slope = a.parts + stat_floats(f);
        a.parts += 2 * stat_floats(f);
    }
    a.splits = key_splits(f, shape);
    return f->dtype == FUSE_BF16 ? launch_shape<__bf16>(shape_of(shape), a, (hipStream_t)stream)
                                 : launch_shape<_Float16>(shape_of(shape), a, (hipStream_t)stream);
}

}  // namespace

extern "C" {

size_t fuse_attention_backward_bytes(const fuse_attn *attn)
{
    return fuse::guard_bytes([&] { return fuse::check_attn(attn) || attn->q_tokens == 0 ? 0 : backward_bytes(attn, nullptr); });
}

size_t fuse_attention_shaped_backward_bytes(const fuse_attn *attn, const fuse_attn_shape *shape)
{
    return fuse::guard_bytes([&] { return fuse::check_attn(attn) || fuse::check_shape(attn, shape) || attn->q_tokens == 0 ? 0 : backward_bytes(attn, shape); });
}

int fuse_attention_zero_rest(const fuse_attn *attn, const fuse_attn_grads *grads, void *stream)
{
    return fuse::guard([&] { return zero_rest_impl(attn, grads, stream); });
}

int fuse_attention_backward(const fuse_attn *attn, const fuse_attn_grads *grads, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return backward_impl(attn, nullptr, grads, workspace, workspace_bytes, stream); });
}

int fuse_attention_shaped_backward(const fuse_attn *attn, const fuse_attn_shape *shape, const fuse_attn_grads *grads, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return backward_impl(attn, shape, grads, workspace, workspace_bytes, stream); });
}

}  // extern "C"
