// Attention over packed sequences, forward: the kernels.  SHAPE (attention.h): what is done to the scores; each set of shapes is
// compiled by a source of its own, side by side.
#pragma once
#include <type_traits>

#include "attention_tiles.h"

namespace fuse {
namespace forward {

constexpr int kRows = 128;                 // rows per tile: 32 per wave
constexpr int kKeys = 64;                  // keys per step
constexpr int kMaxSplits = 64;
constexpr int kJoinBlocks = 8;             // blocks that join a tile's rows: a row for each wave of 32 rows' worth

// Where a call's keys are split: unnormalised results and statistics of every row and split.
struct Parts {
    float *o, *m, *l;                      // (row, split): dim values, maximum, sum
    int splits;                            // 1: not split
};

__device__ __forceinline__ long long part_at(const AttnArgs &a, const Parts &p, long long token, int head, int split)
{
    return (token * a.heads + head) * p.splits + split;
}

// What the scores in registers are multiplied with in the exponent, to base 2.  Capped ones are kept as -r (see Scores): the cap is taken twice, and
// added once to what a row's scores have in common.
template <int SHAPE> constexpr bool kCapOnly = (SHAPE & (kCapped | kSloped)) == kCapped;
template <int SHAPE>
__device__ __forceinline__ float factor_of(const AttnArgs &a)
{
    return kCapOnly<SHAPE> ? 2.0f * a.cap * kLog2e : kScored<SHAPE> ? 1.0f : a.scale * kLog2e;
}

// lse of a row, of the maximum of its scores in registers and the sum of its weights.
template <typename T, int SHAPE>
__device__ __forceinline__ float lse_of(const AttnArgs &a, float m, float l)
{
    if (kCapOnly<SHAPE>)
        return fmaf(m, 2.0f * a.cap, a.cap + log_of<T>(l));
    return fmaf(m, kScored<SHAPE> ? 1.0f / kLog2e : a.scale, log_of<T>(l));
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
//
// Shaped scores: 8192 packed tokens in four sequences, heads as above: plain 266 us, with a cap 287 (two more exponentials' worth per score),
// slopes 265 (an operation each), both 313.  A polynomial for scores within half the cap, instead of the exponential and the division, takes
// as long (293 us where the two took 293).
template <typename T, int DP, int SHAPE>
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
    const int prefix = prefix_of<SHAPE>(a, work.seq), seen = seen_by(a, x, place, prefix);
    const int seen_lo = __builtin_amdgcn_readfirstlane(seen);              // the wave's first row sees least, its last row most
    const int seen_hi = first + wave * 32 < rows ? __builtin_amdgcn_readlane(seen, 31) : 0;

    // this split's keys: begin .. end of those that any row of the tile sees
    int begin = 0, end = seen_by(a, x, place_of(a, min(first + kRows, rows) - 1), prefix);
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
    const Scores<SHAPE> scores(a);
    const float c = factor_of<SHAPE>(a);
    const float slope = SHAPE & kSloped ? a.slopes[head] * kLog2e : 0.0f;

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
                if (kScored<SHAPE>) {
                    const float far = (float)(j + 4 * h - (place + x.nk - x.nq));
                    float d;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        p[i / 16][i % 16] = kCapOnly<SHAPE> ? -scores.turned(p[i / 16][i % 16])
                                                            : scores.of(p[i / 16][i % 16], scores.cap, far + (float)(i / 16 * 32 + 8 * (i % 16 / 4) + i % 4), slope, d);
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
            a.lse[(x.q0 + place) * a.heads + head] = l == 0.0f ? -INFINITY : lse_of<T, SHAPE>(a, m, l);
    }
}

// Joins the splits of every row: a wave per row.  6 to 7 us, most of it the launch.
template <typename T, int SHAPE>
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
        const float w = l == 0.0f ? 0.0f : exp2f((m - top) * factor_of<SHAPE>(a));
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
            a.lse[(x.q0 + place) * a.heads + head] = sum == 0.0f ? -INFINITY : lse_of<T, SHAPE>(a, top, sum);
    }
}

template <typename T, int SHAPE>
int launch(const AttnArgs &a, const Parts &p, unsigned tiles, hipStream_t s)
{
    const unsigned blocks = tiles * a.kv_heads * p.splits;
    if (a.dim <= 64)
        attention_kernel<T, 64, SHAPE><<<blocks, 256, 0, s>>>(a, p);
    else if (a.dim <= 96)
        attention_kernel<T, 96, SHAPE><<<blocks, 256, 0, s>>>(a, p);
    else
        attention_kernel<T, 128, SHAPE><<<blocks, 256, 0, s>>>(a, p);
    int rc = launched("attention_kernel");
    if (rc || p.splits == 1)
        return rc;
    attention_join_kernel<T, SHAPE><<<dim3(tiles * a.kv_heads, kJoinBlocks), 256, 0, s>>>(a, p);
    rc = launched("attention_join_kernel");
    if (!rc)
        set_last_kernel("attention_kernel");
    return rc;
}

#define FUSE_FORWARD(prefix, T, SHAPE) prefix template int launch<T, SHAPE>(const AttnArgs &, const Parts &, unsigned, hipStream_t);

}  // namespace forward
}  // namespace fuse
