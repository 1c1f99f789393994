// Attention over packed sequences, forward (fuse_attention).
#include <type_traits>

#include "attention_tiles.h"

namespace {

using namespace fuse;

constexpr int kRows = 128;                 // rows per tile: 32 per wave
constexpr int kKeys = 64;                  // keys per step
constexpr int kMaxSplits = 64;
constexpr int kJoinBlocks = 8;             // blocks that join a tile's rows: a row for each wave of 32 rows' worth
constexpr float kLog2e = 1.44269504088896340736f;

// Where a call's keys are split: unnormalised results and statistics of every row and split.
struct Parts {
    float *o, *m, *l;                      // (row, split): dim values, maximum, sum
    int splits;                            // 1: not split
};

__device__ __forceinline__ long long part_at(const AttnArgs &a, const Parts &p, long long token, int head, int split)
{
    return (token * a.heads + head) * p.splits + split;
}

// What a column's weights are multiplied with before they are rounded, as a power of two (LIFT), and how many powers of two the maximum
// that they are taken against may lag behind (SLACK).  Every weight is at most 2^(LIFT + SLACK), and the sum, which carries the same factor, is
// at least 2^LIFT.
//
// bf16 has fp32's range: nothing to lift.  fp16 ends at 2^16 and is coarser below 2^-14, so weights take its whole range: those down to
// 2^-25 of the largest one are rounded by half a step of their own value, and smaller ones by 2^-36 of the sum at most.  Unlifted,
// a weight of 2^-25 would be 0, and many of them next to one key that takes almost all of the weight (with a value near 0) are what the
// result is made of.  The slack decides how often results are rescaled: 12288 packed tokens, 32 heads over 8, dim 128, fp16 take 492 us with
// lift 11 and slack 4 as with 7 and 8, 499 us with 13 and 2, 515 us with 15 and 0.
template <typename T> constexpr int kLift = 0;
template <typename T> constexpr int kSlack = 8;
template <> constexpr int kLift<_Float16> = 11;
template <> constexpr int kSlack<_Float16> = 4;

// Running maximum and sum of a column, and its 32 new scores: rescales the result's DT tiles where the maximum has moved.
//
// The maximum that is subtracted is not always the largest score so far: it is moved only when a score's weight is more than 2^SLACK times
// larger, so that most steps leave the results as they are.
template <typename T, int DT>
__device__ __forceinline__ void follow_max(float top, float c, float &m, float &mc, float &l, f32x16 (&o)[DT])
{
    if (!__any((top - m) * c > (float)kSlack<T>))
        return;
    const float next = fmaxf(m, top), to = (next == -INFINITY ? 0.0f : next * c) - (float)kLift<T>;
    const float f = m == -INFINITY ? 0.0f : exp2f(mc - to);
    m = next;
    mc = to;
    l *= f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        o[d] *= f;
}

// log of a sum of lifted weights
template <typename T>
__device__ __forceinline__ float log_of(float sum)
{
    return logf(sum * (1.0f / (1 << kLift<T>)));
}

// One block: 128 rows, 32 per wave as columns (attention_tiles.h), the keys and values that they see in steps of 64 through LDS, loaded
// a step ahead.  One pass: running maximum and sum per column, exp(S - max), rounded, straight into the product with the values.
//
// Bound by how products and vector work share a compute unit: of 12288 packed tokens, 32 heads over 8 of dim 128 (438 GFLOP of what
// is visible) the matrix units are busy for 47 % of the time and the vector units for 52 %, mostly exp (a quarter of the rate of
// other work); 481 us, 0.91 PFLOP/s.  Without its loads the same kernel takes 20 % less; four tiles of 32 KB each way from L2 per step
// and compute unit do not hide entirely behind two blocks.  Tried without gain: the next step's scores among this one's exp
// (500 to 510 us), transposed loads with waits of their own (509), a higher priority for waves in their products (528); blocks of 256
// rows, which read half as much, take 472 us here but lose 4 to 24 % with fewer rows, fewer blocks or a dim of 64.
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 64 ? 3 : 2) attention_kernel(const AttnArgs a, const Parts parts)
{
    using L = Tile<DP>;
    constexpr int kBytes = kKeys * L::kRowBytes;
    __shared__ __attribute__((aligned(256))) char lds[2][2][kBytes];       // [step % 2][K, V]
    __shared__ s16x8 spare[4][2][64];                                      // weights, see add_seen

    const int kvh = blockIdx.x % a.kv_heads;
    const unsigned rest = blockIdx.x / a.kv_heads;
    const int split = rest % parts.splits;
    const Work work = work_of<false>(a, kRows, rest / parts.splits);
    if (!work.any)
        return;
    const Seq &x = work.x;
    const int first = work.first, rows = x.nq * a.group;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int r = first + wave * 32 + (lane & 31);
    const bool in = r < rows;
    const int place = place_of(a, in ? r : rows - 1), head = kvh * a.group + (in ? r : rows - 1) - place * a.group;
    const int seen = seen_by(a, x, place);
    const int seen_lo = __builtin_amdgcn_readfirstlane(seen);              // the wave's first row sees least, its last row most
    const int seen_hi = first + wave * 32 < rows ? __builtin_amdgcn_readlane(seen, 31) : 0;

    // this split's keys: begin .. end of those that any row of the tile sees
    int begin = 0, end = seen_by(a, x, place_of(a, min(first + kRows, rows) - 1));
    if (parts.splits > 1) {
        const int per = ((end + parts.splits - 1) / parts.splits + kKeys - 1) / kKeys * kKeys;
        begin = min(split * per, end);
        end = min(begin + per, end);
    }

    s16x8 q[L::kSteps];
    operands<T, DP>(q, row_of<const T>(a.q, x.q0 + place, head), in, a.dim);
    int row_at[L::kSteps], col_at[L::kCols][2];
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i)
        row_at[i] = L::row_at(lane, i);
#pragma unroll
    for (int i = 0; i < L::kCols; ++i) {
        col_at[i][0] = L::col_at(lane, i, 0);
        col_at[i][1] = L::col_at(lane, i, 1);
    }

    f32x16 o[L::kCols];
    float m, mc, l;
    const float c = a.scale * kLog2e;

    const T *kbase = row_of<const T>(a.k, x.k0, kvh), *vbase = row_of<const T>(a.v, x.k0, kvh);
    const Fill<T, DP, kKeys> fill(a.dim);
    if (a.dim < DP)
        clear_tiles(lds[0][0], sizeof lds);
    auto attend = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        m = -INFINITY, mc = 0.0f, l = 0.0f;
#pragma unroll
        for (int d = 0; d < L::kCols; ++d)
            o[d] = f32x16{};
        if (begin < end) {
            fill.load(lds[0][0], kbase, a.k.token, begin, x.nk);
            fill.load(lds[0][1], vbase, a.v.token, begin, x.nk);
        }
        __syncthreads();
        for (int j = begin, step = 0; j < end; j += kKeys, ++step) {
            const char *kt = lds[step & 1][0], *vt = lds[step & 1][1];
            if (j + kKeys < end) {             // into the tiles that all waves have left behind with the last barrier
                fill.load(lds[(step + 1) & 1][0], kbase, a.k.token, j + kKeys, x.nk);
                fill.load(lds[(step + 1) & 1][1], vbase, a.v.token, j + kKeys, x.nk);
            }
            __builtin_amdgcn_sched_barrier(0); // the loads first, a whole step ahead of the barrier that waits for them
            if (j < seen_hi) {
                f32x16 p[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    p[n] = f32x16{};
#pragma unroll
                    for (int i = 0; i < L::kSteps; ++i)
                        p[n] = product<T>(read_row(kt + n * 32 * L::kRowBytes, row_at[i]), q[i], p[n]);
                }
                const bool masked = j + kKeys > seen_lo;
                if (masked) {
                    const int left = seen - j - 4 * h;
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (n * 32 + 8 * (i / 4) + i % 4 >= left)
                                p[n][i] = -INFINITY;
                }
                float top = p[0][0];
#pragma unroll
                for (int i = 1; i < 32; ++i)
                    top = fmaxf(top, p[i / 16][i % 16]);
                follow_max<T, L::kCols>(both_max(top), c, m, mc, l, o);
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    p[i / 16][i % 16] = __builtin_amdgcn_exp2f(fmaf(p[i / 16][i % 16], c, -mc));
                    l += p[i / 16][i % 16];
                }
                s16x8 w[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    float e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        e[i] = p[n / 2][n % 2 * 8 + i];
                    w[n] = rounded<T>(e);
                }
                if (CAREFUL && masked && holds_no_number<T, DP>(vt, kKeys)) {
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        spare[wave][0][lane] = w[n * 2];
                        spare[wave][1][lane] = w[n * 2 + 1];
                        wave_sees();
                        add_seen<T, DP>(o, vt + n * 32 * L::kRowBytes, spare[wave][0], 64, 32, 0, seen - j - n * 32, 0);
                        wave_sees();
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int d = 0; d < L::kCols; ++d)
                            o[d] = product<T>(read_col(vt + n * 16 * L::kRowBytes, col_at[d][0], col_at[d][1]), w[n], o[d]);
                }
            }
            __syncthreads();
        }
    };
    attend(std::false_type());
    // A masked score is a weight of 0, which the matrix units still multiply with the value: no number where that is not finite.  A
    // block with such a result is done again, with an eye on the values of the steps that have a mask.
    if (any_wave(in && not_finite(o) != 0.0f, lds[0][0]))
        attend(std::true_type());

    l = both_sum(l);
    if (parts.splits > 1) {
        if (in) {
            const long long at = part_at(a, parts, x.q0 + place, head, split);
            if (h == 0) {
                parts.m[at] = m;
                parts.l[at] = l;
            }
#pragma unroll
            for (int d = 0; d < L::kCols; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (d * 32 + i * 8 + h * 4 < a.dim)
                        *reinterpret_cast<f32x4 *>(parts.o + at * a.dim + d * 32 + i * 8 + h * 4) =
                            f32x4{o[d][i * 4], o[d][i * 4 + 1], o[d][i * 4 + 2], o[d][i * 4 + 3]};
        }
        return;
    }

    const float f = l > 0.0f ? 1.0f / l : 0.0f;        // (no key seen: 0; a score that is no number: o holds none either)
    if (in) {
        write_columns<T>(o, f, row_of<T>(a.out, x.q0 + place, head), h, a.dim);
        if (a.lse && h == 0)
            a.lse[(x.q0 + place) * a.heads + head] = l == 0.0f ? -INFINITY : fmaf(m, a.scale, log_of<T>(l));
    }
}

// Joins the splits of every row: a wave per row.  6 to 7 us, most of it the launch.
template <typename T>
__global__ void __launch_bounds__(256) attention_join_kernel(const AttnArgs a, const Parts parts)
{
    const int kvh = blockIdx.x % a.kv_heads;
    const Work work = tile_at<false>(a, kRows, blockIdx.x / a.kv_heads);
    const Seq &x = work.x;
    const int rows = work.any ? min(work.first + kRows, x.nq * a.group) : 0, lane = threadIdx.x & 63;
    for (int r = work.first + blockIdx.y * 4 + (threadIdx.x >> 6); r < rows; r += 4 * kJoinBlocks) {
        const int place = place_of(a, r), head = kvh * a.group + r - place * a.group;
        const long long at = part_at(a, parts, x.q0 + place, head, 0);
        const bool mine = lane < parts.splits;
        const float m = mine ? parts.m[at + lane] : -INFINITY, l = mine ? parts.l[at + lane] : 0.0f;
        float top = m;
#pragma unroll
        for (int i = 32; i > 0; i >>= 1)
            top = fmaxf(top, __shfl_xor(top, i, 64));
        const float w = l == 0.0f ? 0.0f : exp2f((m - top) * (a.scale * kLog2e));
        const float sum = wave_sum(w * l);
        float o0 = 0.0f, o1 = 0.0f;
        // eight splits' loads in flight, without a branch around them: one by one, 64 splits took 35 us
        const float *o = parts.o + at * a.dim;
        const int d0 = min(lane, a.dim - 1), d1 = min(lane + 64, a.dim - 1);
        for (int i = 0; i < parts.splits; i += 8) {
            float v0[8], v1[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int k = min(i + u, parts.splits - 1);
                v0[u] = o[(long long)k * a.dim + d0];
                v1[u] = o[(long long)k * a.dim + d1];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u < parts.splits) {                                // (its weight would be 0, but not 0 times what is not finite)
                    const float f = __shfl(w, i + u, 64);
                    o0 = fmaf(f, v0[u], o0);
                    o1 = fmaf(f, v1[u], o1);
                }
        }
        const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
        T *out = row_of<T>(a.out, x.q0 + place, head);
        if (lane < a.dim)
            out[lane] = (T)(o0 * f);
        if (lane + 64 < a.dim)
            out[lane + 64] = (T)(o1 * f);
        if (a.lse && lane == 0)
            a.lse[(x.q0 + place) * a.heads + head] = sum == 0.0f ? -INFINITY : fmaf(top, a.scale, log_of<T>(sum));
    }
}

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
int launch(const AttnArgs &a, const Parts &p, unsigned tiles, hipStream_t s)
{
    const unsigned blocks = tiles * a.kv_heads * p.splits;
    if (a.dim <= 64)
        attention_kernel<T, 64><<<blocks, 256, 0, s>>>(a, p);
    else if (a.dim <= 96)
        attention_kernel<T, 96><<<blocks, 256, 0, s>>>(a, p);
    else
        attention_kernel<T, 128><<<blocks, 256, 0, s>>>(a, p);
    int rc = launched("attention_kernel");
    if (rc || p.splits == 1)
        return rc;
    attention_join_kernel<T><<<dim3(tiles * a.kv_heads, kJoinBlocks), 256, 0, s>>>(a, p);
    rc = launched("attention_join_kernel");
    if (!rc)
        set_last_kernel("attention_kernel");
    return rc;
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
    if (f->q_tokens == 0 || f->seqs == 0)
        return FUSE_OK;
    AttnArgs a = attn_args(f);
    a.out = {out, out_token_ld, out_head_ld};
    a.lse = lse;
    Parts p = {};
    p.splits = splits_of(f);
    const size_t need = parts_floats(f, p.splits) * sizeof(float);
    if (need && (!workspace || !on_16_bytes(workspace) || workspace_bytes < need))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(need) + " bytes on 16 are needed");
    p.o = static_cast<float *>(workspace);
    p.m = p.o + (size_t)f->q_tokens * f->heads * p.splits * f->dim;
    p.l = p.m + (size_t)f->q_tokens * f->heads * p.splits;
    const unsigned tiles = (unsigned)tiles_of(f);
    return f->dtype == FUSE_BF16 ? launch<__bf16>(a, p, tiles, (hipStream_t)stream) : launch<_Float16>(a, p, tiles, (hipStream_t)stream);
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
    if (fuse::check_attn(attn))
        return 0;
    return parts_floats(attn, splits_of(attn)) * sizeof(float);
}

int fuse_attention(const fuse_attn *attn, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return attention_impl(attn, out, out_token_ld, out_head_ld, lse, workspace, workspace_bytes, stream); });
}

}  // extern "C"
