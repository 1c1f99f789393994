// Attention over packed sequences, gradients (fuse_attention_backward).
#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"

namespace {

using namespace fuse;

constexpr int kRows = 128;                 // rows per block: 32 per wave
constexpr int kStep = 64;                  // keys, or rows, per step
constexpr int kKeys = 64;                  // keys per block of their kernel
constexpr int kJoinBlocks = 4;             // blocks that join a tile's splits
constexpr float kLog2e = 1.44269504088896340736f;

// fp16: P and dS = P o (dP - delta) are multiplied with powers of two before they are rounded, and their products with the inverse.  P is some
// 1 / keys and gradients are small, so dS as it is falls among the numbers below 2^-14, of which fp16 keeps few digits (below 2^-25 none);
// and large gradients leave its range at 2^16.  bf16 has fp32's range.
//   queries: a column's lift begins high and goes down, with the sums so far, when one of its dS would pass 2^15: to between 2^11 and 2^12,
//            so that it seldom moves again.  dS is rounded by half a step of its own value down to 2^-25 of the column's largest, and by 2^-36
//            of the largest below that.
//   keys:    P by 2^15; dS by the least lift of the rows that the block reads, which the queries' kernel leaves for every 32 rows.
// A whole backward pass in fp16, without and with this: 8192 packed tokens, 32 heads over 8, dim 128: 761 and 779 us; 3331 tokens, 12 heads
// over 4, dim 80: 66 and 69 us.
template <typename T> constexpr bool kLifted = false;
template <> constexpr bool kLifted<_Float16> = true;
constexpr int kMostLift = 60;              // 2^60 dS of the first keys stay within fp32: |dP| is below 2^40
constexpr int kLiftP = 15;

// Lowers a column's lift if one of its 16 new dS, which carry it already, passes 2^15; the sums so far go with it.
template <int DT>
__device__ __forceinline__ void lower(float (&w)[16], int &lift, f32x16 (&o)[DT])
{
    float top = fabsf(w[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i)
        top = fmaxf(top, fabsf(w[i]));
    if (!__any(both_max(top) > 32768.0f))
        return;
    top = 0.0f;                            // the largest of those that are numbers
#pragma unroll
    for (int i = 0; i < 16; ++i)
        top = fabsf(w[i]) < INFINITY ? fmaxf(top, fabsf(w[i])) : top;
    top = both_max(top);
    const bool over = top > 32768.0f;
    const int down = over ? __builtin_amdgcn_frexp_expf(top) - 12 : 0;     // (to between 2^11 and 2^12)
    const float f = ldexpf(1.0f, -down);
    lift -= down;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        w[i] *= f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        o[d] *= f;
}

// Gradient of the queries, and delta and lse, in the order of the rows, for the keys' kernel.  As the forward kernel: 32 rows per wave
// as columns, keys and values step by step through LDS; the keys are read twice, as rows for S and transposed for t(K) t(dS).
//
// Scores are taken twice, here and for the keys: one kernel for all three gradients would have to add up those of the queries over
// blocks of keys, by atomics in an order that changes or through memory.  8192 packed tokens, 32 heads over 8 of dim 128: 297 us here
// (three products, 0.94 PFLOP/s) and 420 us for the keys (four products, 0.89 PFLOP/s).
template <typename T, int DP>
__global__ void __launch_bounds__(256, 2) attention_query_grad_kernel(const AttnArgs a)
{
    using L = Tile<DP>;
    constexpr int kBytes = kStep * L::kRowBytes;
    __shared__ __attribute__((aligned(256))) char lds[2][2][kBytes];       // [step % 2][K, V]
    __shared__ s16x8 spare[4][2][64];                                      // weights, see add_seen

    const int kvh = blockIdx.x % a.kv_heads;
    const Work work = work_of<false>(a, kRows, blockIdx.x / a.kv_heads);
    if (!work.any)
        return;
    const Seq &x = work.x;
    const int first = work.first, rows = x.nq * a.group;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int r = first + wave * 32 + (lane & 31);
    const bool in = r < rows;
    const int place = place_of(a, in ? r : rows - 1), head = kvh * a.group + (in ? r : rows - 1) - place * a.group;
    const int seen = seen_by(a, x, place);
    const int seen_lo = __builtin_amdgcn_readfirstlane(seen);
    const int seen_hi = first + wave * 32 < rows ? __builtin_amdgcn_readlane(seen, 31) : 0;
    const int end = seen_by(a, x, place_of(a, min(first + kRows, rows) - 1));

    s16x8 q[L::kSteps], g[L::kSteps];
    operands<T, DP>(q, row_of<const T>(a.q, x.q0 + place, head), in, a.dim);
    operands<T, DP>(g, row_of<const T>(a.dout, x.q0 + place, head), in, a.dim);
    float delta = 0.0f, lse2 = 0.0f;
    {
        typedef T t8 __attribute__((ext_vector_type(8)));
        s16x8 o[L::kSteps];
        operands<T, DP>(o, row_of<const T>(a.out, x.q0 + place, head), in, a.dim);
#pragma unroll
        for (int i = 0; i < L::kSteps; ++i) {
            const t8 u = __builtin_bit_cast(t8, g[i]), v = __builtin_bit_cast(t8, o[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = fmaf((float)u[e], (float)v[e], delta);
        }
        delta = both_sum(delta);
    }
    if (in) {
        const long long at = stat_at(a, x.q0 + place, head);
        lse2 = a.lse[(x.q0 + place) * a.heads + head] * kLog2e;
        if (h == 0) {
            a.delta[at] = delta;
            a.lse2[at] = kLifted<T> ? lse2 - kLiftP : lse2;
        }
    }

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
    int lift = 0;
    const float c = a.scale * kLog2e;

    const T *kbase = row_of<const T>(a.k, x.k0, kvh), *vbase = row_of<const T>(a.v, x.k0, kvh);
    const Fill<T, DP, kStep> fill(a.dim);
    if (a.dim < DP)
        clear_tiles(lds[0][0], sizeof lds);
    auto sum_up = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int d = 0; d < L::kCols; ++d)
            o[d] = f32x16{};
        if (kLifted<T>)
            lift = kMostLift;
        if (end > 0) {
            fill.load(lds[0][0], kbase, a.k.token, 0, x.nk);
            fill.load(lds[0][1], vbase, a.v.token, 0, x.nk);
        }
        __syncthreads();
        for (int j = 0, step = 0; j < end; j += kStep, ++step) {
            const char *kt = lds[step & 1][0], *vt = lds[step & 1][1];
            if (j + kStep < end) {
                fill.load(lds[(step + 1) & 1][0], kbase, a.k.token, j + kStep, x.nk);
                fill.load(lds[(step + 1) & 1][1], vbase, a.v.token, j + kStep, x.nk);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (j < seen_hi) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    f32x16 p = {}, dp = {};
#pragma unroll
                    for (int i = 0; i < L::kSteps; ++i) {
                        p = product<T>(read_row(kt + n * 32 * L::kRowBytes, row_at[i]), q[i], p);
                        dp = product<T>(read_row(vt + n * 32 * L::kRowBytes, row_at[i]), g[i], dp);
                    }
                    float w[16];
                    const float from = kLifted<T> ? (float)lift - lse2 : -lse2;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        w[i] = __builtin_amdgcn_exp2f(fmaf(p[i], c, from)) * (dp[i] - delta);
                    const bool masked = j + kStep > seen_lo;
                    if (masked) {
                        const int left = seen - j - n * 32 - 4 * h;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (8 * (i / 4) + i % 4 >= left)
                                w[i] = 0.0f;
                    }
                    if (kLifted<T>)
                        lower(w, lift, o);
                    const s16x8 ds[2] = {rounded<T>(w), rounded<T>(w + 8)};
                    if (CAREFUL && masked && holds_no_number<T, DP>(kt + n * 32 * L::kRowBytes, 32)) {
                        spare[wave][0][lane] = ds[0];
                        spare[wave][1][lane] = ds[1];
                        wave_sees();
                        add_seen<T, DP>(o, kt + n * 32 * L::kRowBytes, spare[wave][0], 64, 32, 0, seen - j - n * 32, 0);
                        wave_sees();
                    } else {
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int d = 0; d < L::kCols; ++d)
                                o[d] = product<T>(read_col(kt + (n * 2 + u) * 16 * L::kRowBytes, col_at[d][0], col_at[d][1]), ds[u], o[d]);
                    }
                }
            }
            __syncthreads();
        }
    };
    sum_up(std::false_type());
    if (any_wave(in && not_finite(o) != 0.0f, lds[0][0]))     // as in the forward kernel: 0 for a masked key, times a key that is not finite
        sum_up(std::true_type());

    if (in)
        write_columns<T>(o, kLifted<T> ? ldexpf(a.scale, -lift) : a.scale, row_of<T>(a.dq, x.q0 + place, head), h, a.dim);
    if (kLifted<T> && first + wave * 32 < rows) {
#pragma unroll
        for (int i = 16; i > 0; i >>= 1)
            lift = min(lift, __shfl_xor(lift, i, 64));
        if (lane == 0)
            a.lifts[lift_at(a, work, kvh, first + wave * 32)] = lift;
    }
}

// Gradients of the keys and values: 64 keys per block, the rows that see them step by step through LDS, all query heads of the key
// head among them.  Both tiles are read twice, as rows (S and dP) and transposed (t(dout) P and t(Q) dS).
//
// Two waves share 32 keys, as columns.  Each takes half of a step's rows for S, dP, P and dS, the two exchange P and dS through LDS, and
// each adds all rows' products to half of the dims of dV and dK.  That is the same work as a wave for itself, but 64 registers of sums
// instead of 128: with those, next to 64 of keys and values, nothing is left to load operands ahead of the products.  For a dim of 128 all 256
// registers are taken and 16 to 20 bytes per lane are in scratch memory.
//
// EVEN: the rows of one pass of a tile's loads are whole tokens (the group divides their number), so they lie the same distance from
// the next pass's and their addresses are scalars with 32 bit offsets per lane: 481 against 521 us for a group of four.  Else, and where
// heads or tokens are far apart, every row's place is divided out (the two in one kernel: 78 against 68 us for a group of three).
template <typename T, int DP, bool EVEN>
__global__ void __launch_bounds__(256, 2) attention_key_grad_kernel(const AttnArgs a)
{
    using L = Tile<DP>;
    constexpr int kBytes = kStep * L::kRowBytes, kHalfCols = (L::kCols + 1) / 2;
    __shared__ __attribute__((aligned(256))) char lds[2][2][kBytes];       // [step % 2][Q, dout]
    __shared__ s16x8 exchange[2][2][2][2][64];                             // [keys][rows' half][16 rows][P, dS][lane]
    // (80 KB for a dim of 128: two blocks per compute unit, whose steps overlap)

    const int kvh = blockIdx.x % a.kv_heads;
    const unsigned rest = blockIdx.x / a.kv_heads;
    const int split = rest % a.splits;
    const Work tile = work_of<true>(a, kKeys, rest / a.splits);
    if (!tile.any)
        return;
    const Seq &x = tile.x;
    const int first = tile.first;

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), keys = wave & 1, half = wave >> 1;
    const int key0 = first + keys * 32, key = key0 + (lane & 31);
    const bool in = key < x.nk;
    // the rows that see a key: from row from(key) on; this split's steps: rows begin .. of those that any key of the tile has
    const int rows = x.nq * a.group, seen = first_that_sees(a, x, first) * a.group;
    const int steps = (rows - seen + kStep - 1) / kStep, per = (steps + a.splits - 1) / a.splits;
    const int begin = seen + min(split * per, steps) * kStep, last = seen + (min((split + 1) * per, steps) - 1) * kStep;
    const int from = first_that_sees(a, x, min(key, x.nk - 1)) * a.group;
    const int from_lo = key0 < x.nk ? __builtin_amdgcn_readfirstlane(from) : rows;
    const int from_hi = __builtin_amdgcn_readlane(from, 31);

    s16x8 k[L::kSteps], v[L::kSteps];
    operands<T, DP>(k, row_of<const T>(a.k, x.k0 + min(key, x.nk - 1), kvh), in, a.dim);
    operands<T, DP>(v, row_of<const T>(a.v, x.k0 + min(key, x.nk - 1), kvh), in, a.dim);
    int row_at[L::kSteps], col_at[kHalfCols][2];
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i)
        row_at[i] = L::row_at(lane, i);
#pragma unroll
    for (int i = 0; i < kHalfCols; ++i) {
        col_at[i][0] = L::col_at(lane, half * kHalfCols + i, 0);
        col_at[i][1] = L::col_at(lane, half * kHalfCols + i, 1);
    }
    f32x16 dk[kHalfCols], dv[kHalfCols];
    const float c = a.scale * kLog2e;

    const T *qbase = row_of<const T>(a.q, x.q0, kvh * a.group), *gbase = row_of<const T>(a.dout, x.q0, kvh * a.group);
    const long long sbase = stat_at(a, x.q0, kvh * a.group);
    const Fill<T, DP, kStep> fill(a.dim);
    const int tokens = fill.kPerPass / a.group, lane_place = place_of(a, fill.row), lane_head = fill.row - lane_place * a.group;
    const unsigned qlane = fill.lane_of(lane_place * a.q.token + lane_head * a.q.head);
    const unsigned glane = fill.lane_of(lane_place * a.dout.token + lane_head * a.dout.head);
    auto load = [&](int b, int r0) {
        if (EVEN && r0 + kStep <= rows) {
            const int p = place_of(a, r0);
            fill.load_whole(lds[b][0], qbase + p * a.q.token, qlane, tokens * a.q.token);
            fill.load_whole(lds[b][1], gbase + p * a.dout.token, glane, tokens * a.dout.token);
            return;
        }
        fill.load(lds[b][0], r0, rows, [&](int r) {
            const int p = place_of(a, r);
            return qbase + p * a.q.token + (r - p * a.group) * a.q.head;
        });
        fill.load(lds[b][1], r0, rows, [&](int r) {
            const int p = place_of(a, r);
            return gbase + p * a.dout.token + (r - p * a.group) * a.dout.head;
        });
    };
    int lift = 0;
    if (kLifted<T>) {
        lift = kMostLift;
        for (int r = begin / 32 * 32 + threadIdx.x * 32; r < min(last + kStep, rows); r += 256 * 32)
            lift = min(lift, a.lifts[lift_at(a, tile, kvh, r)]);
        lift = least_of_block(lift, lds[0][0]);
    }
    const float lift_ds = kLifted<T> ? ldexpf(1.0f, lift - kLiftP) : 1.0f;   // (w carries kLiftP already)
    if (a.dim < DP)
        clear_tiles(lds[0][0], sizeof lds);
    auto sum_up = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int d = 0; d < kHalfCols; ++d)
            dk[d] = dv[d] = f32x16{};
        // from the last rows down: blocks that run at the same time see different first rows, but all of a sequence's last ones, so
        // each step's tiles are in L2 for all of them (from the first rows up, half of what is read comes from behind it)
        if (begin <= last)
            load(0, last);
        __syncthreads();
        for (int r0 = last, B = 0; r0 >= begin; r0 -= kStep, B ^= 1) {
            const char *qt = lds[B][0], *gt = lds[B][1];
            const bool work = r0 + half * 32 + 32 > from_lo;
            f32x4u lse[4], delta[4];           // of rows 8 i + 4 h ..; behind the last row they are anything, and masked
            if (work) {
                const long long at = sbase + r0 + half * 32 + 4 * h;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lse[i] = *reinterpret_cast<const f32x4u *>(a.lse2 + at + 8 * i);
                    delta[i] = *reinterpret_cast<const f32x4u *>(a.delta + at + 8 * i);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (r0 > begin)
                load(B ^ 1, r0 - kStep);
            __builtin_amdgcn_sched_barrier(0);
            if (work) {
                f32x16 p = {}, dp = {};
#pragma unroll
                for (int i = 0; i < L::kSteps; ++i) {
                    p = product<T>(read_row(qt + half * 32 * L::kRowBytes, row_at[i]), k[i], p);
                    dp = product<T>(read_row(gt + half * 32 * L::kRowBytes, row_at[i]), v[i], dp);
                }
                ahead<L::kSteps * 2, 6>();
                float w[16], ds[16];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        w[i * 4 + u] = __builtin_amdgcn_exp2f(fmaf(p[i * 4 + u], c, -lse[i][u]));
                        ds[i * 4 + u] = w[i * 4 + u] * (dp[i * 4 + u] - delta[i][u]);
                        if (kLifted<T>)
                            ds[i * 4 + u] *= lift_ds;
                    }
                }
                if (r0 + half * 32 < from_hi || r0 + half * 32 + 32 > rows) {
                    const int skip = from - r0 - half * 32 - 4 * h, left = rows - r0 - half * 32 - 4 * h;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (8 * (i / 4) + i % 4 < skip || 8 * (i / 4) + i % 4 >= left)
                            w[i] = ds[i] = 0.0f;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    exchange[keys][half][u][0][lane] = rounded<T>(w + u * 8);
                    exchange[keys][half][u][1][lane] = rounded<T>(ds + u * 8);
                }
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < 2; ++n)
                if (r0 + n * 32 + 32 > from_lo) {
                    const char *qn = qt + n * 32 * L::kRowBytes, *gn = gt + n * 32 * L::kRowBytes;
                    const bool masked = r0 + n * 32 < from_hi || r0 + n * 32 + 32 > rows;
                    if (CAREFUL && masked && (holds_no_number<T, DP>(qn, 32) || holds_no_number<T, DP>(gn, 32))) {
                        const int low = from - r0 - n * 32, high = rows - r0 - n * 32;
                        add_seen<T, DP>(dv, gn, exchange[keys][n][0][0], 2 * 64, 32, low, high, half * kHalfCols);
                        add_seen<T, DP>(dk, qn, exchange[keys][n][0][1], 2 * 64, 32, low, high, half * kHalfCols);
                        continue;
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const s16x8 bp = exchange[keys][n][u][0][lane], bs = exchange[keys][n][u][1][lane];
                        const int at = u * 16 * L::kRowBytes;
#pragma unroll
                        for (int d = 0; d < kHalfCols; ++d)
                            if (L::kCols % 2 == 0 || half * kHalfCols + d < L::kCols) {
                                dv[d] = product<T>(read_col(gn + at, col_at[d][0], col_at[d][1]), bp, dv[d]);
                                dk[d] = product<T>(read_col(qn + at, col_at[d][0], col_at[d][1]), bs, dk[d]);
                            }
                    }
                }
            __syncthreads();
        }
    };
    sum_up(std::false_type());
    if (any_wave(in && not_finite(dk) + not_finite(dv) != 0.0f, lds[0][0]))   // 0 for a masked row, times a row that is not finite
        sum_up(std::true_type());

    const int d0 = half * kHalfCols * 32;
    const float fk = kLifted<T> ? ldexpf(a.scale, -lift) : a.scale, fv = kLifted<T> ? 1.0f / (1 << kLiftP) : 1.0f;
    if (in && a.splits > 1) {
        float *part = a.parts + (((x.k0 + key) * a.kv_heads + kvh) * a.splits + split) * 2 * a.dim + d0;
        write_columns<float>(dk, fk, part, h, a.dim - d0);
        write_columns<float>(dv, fv, part + a.dim, h, a.dim - d0);
    } else if (in) {
        write_columns<T>(dk, fk, row_of<T>(a.dk, x.k0 + key, kvh) + d0, h, a.dim - d0);
        write_columns<T>(dv, fv, row_of<T>(a.dv, x.k0 + key, kvh) + d0, h, a.dim - d0);
    }
}

// Adds the splits of the keys' and values' gradients, in order.
template <typename T>
__global__ void __launch_bounds__(256) attention_key_join_kernel(const AttnArgs a)
{
    const int kvh = blockIdx.x % a.kv_heads;
    const Work tile = tile_at<true>(a, kKeys, blockIdx.x / a.kv_heads);
    if (!tile.any)
        return;
    const int quads = a.dim / 4, all = min(kKeys, tile.x.nk - tile.first) * 2 * quads;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < all; i += 256 * kJoinBlocks) {
        const int d = i % quads * 4, which = i / quads & 1;
        const long long token = tile.x.k0 + tile.first + i / quads / 2;
        const float *part = a.parts + ((token * a.kv_heads + kvh) * a.splits * 2 + which) * a.dim + d;
        f32x4 sum = {};
        for (int s = 0; s < a.splits; s += 4) {
            f32x4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = *reinterpret_cast<const f32x4 *>(part + (long long)min(s + u, a.splits - 1) * 2 * a.dim);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (s + u < a.splits)
                    sum += v[u];
        }
        typedef T t4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<t4 *>(row_of<T>(which ? a.dv : a.dk, token, kvh) + d) = t4{(T)sum[0], (T)sum[1], (T)sum[2], (T)sum[3]};
    }
}

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
int key_splits(const fuse_attn *f)
{
    if (f->seqs == 0)
        return 1;
    const long long blocks = first_tile(f->k_tokens, (int)f->seqs, kKeys) * f->kv_heads;
    const long long steps = f->q_tokens * (f->heads / f->kv_heads) / f->seqs / kStep / 2;
    const long long n = std::min(1280 / blocks, steps / 3);
    return (int)(n < 1 ? 1 : n > 32 ? 32 : n);
}

// delta and lse2, each with room for a last step's rows behind the last row, and the splits' sums
size_t stat_floats(const fuse_attn *f) { return ((size_t)f->q_tokens * f->heads + kStep + 3) / 4 * 4; }
// (fp16) the lifts
size_t lift_ints(const fuse_attn *f)
{
    return f->dtype == FUSE_F16 ? ((size_t)first_tile(f->q_tokens * (f->heads / f->kv_heads), (int)f->seqs, 32) * f->kv_heads + 3) / 4 * 4 : 0;
}
size_t backward_bytes(const fuse_attn *f)
{
    const int splits = key_splits(f);
    return (stat_floats(f) * 2 + lift_ints(f) + (splits > 1 ? (size_t)f->k_tokens * f->kv_heads * splits * 2 * f->dim : 0)) * sizeof(float);
}

template <typename T, int DP>
int launch_keys(const AttnArgs &a, unsigned blocks, hipStream_t s)
{
    // (a pass's rows are 32 bit offsets in bytes from its first)
    const bool near = std::max(std::max(a.q.token, a.q.head), std::max(a.dout.token, a.dout.head)) <= 1 << 25;
    if (near && Fill<T, DP, kStep>::kPerPass % a.group == 0)
        attention_key_grad_kernel<T, DP, true><<<blocks, 256, 0, s>>>(a);
    else
        attention_key_grad_kernel<T, DP, false><<<blocks, 256, 0, s>>>(a);
    return launched("attention_key_grad_kernel");
}

template <typename T, int DP>
int launch_dim(const AttnArgs &a, hipStream_t s)
{
    const long long q_tiles = first_tile(a.q_tokens * a.group, a.seqs, kRows), k_tiles = first_tile(a.k_tokens, a.seqs, kKeys);
    if (a.q_tokens > 0) {
        attention_query_grad_kernel<T, DP><<<(unsigned)(q_tiles * a.kv_heads), 256, 0, s>>>(a);
        if (const int rc = launched("attention_query_grad_kernel"))
            return rc;
    }
    if (a.k_tokens == 0)
        return FUSE_OK;
    const unsigned blocks = (unsigned)(k_tiles * a.kv_heads);
    if (a.splits > 1) {
        if (const int rc = launch_keys<T, DP>(a, blocks * a.splits, s))
            return rc;
        attention_key_join_kernel<T><<<dim3(blocks, kJoinBlocks), 256, 0, s>>>(a);
        const int rc = launched("attention_key_join_kernel");
        if (!rc)
            set_last_kernel("attention_key_grad_kernel");
        return rc;
    }
    return launch_keys<T, DP>(a, blocks, s);
}

template <typename T>
int launch_grads(const AttnArgs &a, hipStream_t s)
{
    return a.dim <= 64 ? launch_dim<T, 64>(a, s) : a.dim <= 96 ? launch_dim<T, 96>(a, s) : launch_dim<T, 128>(a, s);
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
    AttnArgs a = grad_args(f, g);
    a.dout = {const_cast<void *>(g->dout), g->dout_token_ld, g->dout_head_ld};
    a.out = {const_cast<void *>(g->out), g->out_token_ld, g->out_head_ld};
    a.lse = const_cast<float *>(g->lse);
    a.delta = static_cast<float *>(workspace);
    a.lse2 = a.delta + stat_floats(f);
    a.lifts = reinterpret_cast<int *>(a.lse2 + stat_floats(f));
    a.parts = a.lse2 + stat_floats(f) + lift_ints(f);
    a.splits = key_splits(f);
    return f->dtype == FUSE_BF16 ? launch_grads<__bf16>(a, (hipStream_t)stream) : launch_grads<_Float16>(a, (hipStream_t)stream);
}

}  // namespace

extern "C" {

size_t fuse_attention_backward_bytes(const fuse_attn *attn)
{
    return fuse::check_attn(attn) || attn->q_tokens == 0 ? 0 : backward_bytes(attn);
}

int fuse_attention_zero_rest(const fuse_attn *attn, const fuse_attn_grads *grads, void *stream)
{
    return fuse::guard([&] { return zero_rest_impl(attn, grads, stream); });
}

int fuse_attention_backward(const fuse_attn *attn, const fuse_attn_grads *grads, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return backward_impl(attn, grads, workspace, workspace_bytes, stream); });
}

}  // extern "C"
