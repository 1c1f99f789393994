// A cache of keys and values in 8 bits on pages (fuse_cache_write), and attention over it (fuse_attention_cache).
//
// Every place of the cache and key head has a row of `dim` values of e4m3 and a scale in fp32:  x = scale * value,
//   scale = max(|x|_max, 2^-100) / 448,  value = x / scale, rounded to nearest, ties to even.
#include <algorithm>

#include "attention_tiles.h"

namespace {

using namespace fuse;

typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr float kMostE4m3 = 448.0f;
constexpr float kLeastMax = 0x1p-100f;     // so that neither a scale nor its inverse leaves fp32's normal range

// r / d for r < 2^31, exact (see place_of).
struct Divider {
    unsigned d, mul, shift;
};
__device__ __forceinline__ int quotient(const Divider &v, int r) { return v.d == 1 ? r : (int)(__umulhi((unsigned)r, v.mul) >> v.shift); }
Divider divider(unsigned d)
{
    int n = 0;
    while (((uint64_t)1 << n) < d)
        ++n;
    return {d, (unsigned)(((uint64_t)1 << (31 + n)) / d + 1), n > 0 ? (unsigned)n - 1 : 0};
}

struct Pages {
    unsigned char *k, *v;
    float *k_scale, *v_scale;
    long long page_ld, head_ld, place_ld;  // bytes
    long long scale_page_ld, scale_head_ld;
    const int *table;
    long long table_ld;
    int count, width;                      // pages; entries of a sequence's table
    Divider size;                          // places per page
};

struct CacheArgs {
    Mat q, out;
    Mat k, v;                              // writing: rows that go into the cache
    float *lse;
    Pages pages;
    float *parts;                          // (row, split): dim values; then maxima, then sums
    const void *q_off, *lengths;
    const long long *tree;
    const float *slopes;
    long long q_tokens;
    int seqs, heads, kv_heads, group, dim, causal, off64, splits;
    int tile;                              // rows of a block
    float scale, cap;
    Divider by_group;
    Divider by_row;                        // writing: rows of a token
};

// Sequence s: its new tokens, and its keys that have a place; k0 is that of the first new token (also where that is before the first place, or
// behind the last one that the table has).
__device__ __forceinline__ Seq seq_at(const CacheArgs &a, int s)
{
    Seq x;
    const long long q0 = offset_at(a.q_off, s, a.off64), q1 = offset_at(a.q_off, s + 1, a.off64);
    const long long room = (long long)a.pages.width * a.pages.size.d;      // (below 2^31 - 4096, which the host checks)
    x.q0 = min(max(q0, 0LL), a.q_tokens);
    x.nq = (int)(min(max(q1, x.q0), a.q_tokens) - x.q0);
    const long long keys = min(max(offset_at(a.lengths, s, a.off64), 0LL), (1LL << 31) - 4096);
    x.k0 = keys - x.nq;
    x.nk = (int)min(keys, room);
    return x;
}

// ----------------------------------------------------------------------------------- writing ---

constexpr int kWriteTokens = 8;            // per block

// Larger of two, and no number if either is none.
__device__ __forceinline__ float max_or_nan(float a, float b) { return a >= b || a != a ? a : b; }

// Keys and values of new tokens into the cache: sixteen lanes per row, 16 bytes of it each, four rows of a lane in flight.  Bound by memory: a
// row is read and written once.  24576 tokens, 8 heads of dim 128, 153 MB: 36 us (4.2 TB/s); 43 us with one row of a lane in flight, 40
// with eight; blocks of 4, 16 and 32 tokens take 37, 41 and 49.  value = (448 x) / max: 448 x is exact in fp32 (both are taken 2^-10 times, within its range), and the
// quotient is corrected to the last bit, so that ties are ties.
template <typename T>
__global__ void __launch_bounds__(256) cache_write_kernel(const CacheArgs a)
{
    constexpr int kAtOnce = 4;
    typedef T t8 __attribute__((ext_vector_type(8)));
    const Work w = tile_at<false>(a, kWriteTokens, blockIdx.x);
    if (!w.any)
        return;
    const Pages &g = a.pages;
    const int rows = min(kWriteTokens, w.x.nq - w.first) * 2 * a.kv_heads, chunk = threadIdx.x & 15;
    const bool in = chunk * 8 < a.dim;
    for (int r0 = threadIdx.x >> 4; r0 < rows; r0 += 16 * kAtOnce) {
        t8 x8[kAtOnce];
        int head[kAtOnce], page[kAtOnce], within[kAtOnce];                 // page -1: no such place
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int r = r0 + u * 16, t = quotient(a.by_row, r), place = (int)w.x.k0 + w.first + t;
            head[u] = (r - t * 2 * a.kv_heads) >> 1;
            page[u] = -1;
            x8[u] = t8{};
            if (r < rows && place >= 0 && place < w.x.nk) {
                const int n = quotient(g.size, place);
                page[u] = g.table[w.seq * g.table_ld + n];
                within[u] = place - n * (int)g.size.d;
                if (in)
                    x8[u] = *reinterpret_cast<const t8 *>(row_of<const T>(r & 1 ? a.v : a.k, w.x.q0 + w.first + t, head[u]) + chunk * 8);
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (page[u] < 0 || page[u] >= g.count)
                continue;
            const bool value = r0 & 1;                                     // (rows of a lane are an even number apart)
            float x[8], top = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = (float)x8[u][i];
                top = max_or_nan(top, fabsf(x[i]));
            }
            top = max_or_nan(top, moved<0xB1>(top));
            top = max_or_nan(top, moved<0x4E>(top));
            top = max_or_nan(top, moved<0x141>(top));
            top = max_or_nan(top, moved<0x140>(top));
            const bool fine = top < INFINITY;                              // else the scale is no number, and so is all that is made of the row
            top = fine ? fmaxf(top, kLeastMax) : 1.0f;
            const float part = top * 0x1p-10f, inv = 1.0f / part;
            int bits[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float q[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float y = fine ? x[i + e] * (kMostE4m3 * 0x1p-10f) : 0.0f, about = y * inv;
                    q[e] = fmaf(fmaf(-about, part, y), inv, about);
                }
                if (i % 4 == 0)
                    bits[i / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], bits[i / 4], false);
                else
                    bits[i / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], bits[i / 4], true);
            }
            if (in)
                *reinterpret_cast<uint2 *>((value ? g.v : g.k) + page[u] * g.page_ld + head[u] * g.head_ld + within[u] * g.place_ld + chunk * 8) =
                    make_uint2(bits[0], bits[1]);
            if (chunk == 0)
                (value ? g.v_scale : g.k_scale)[page[u] * g.scale_page_ld + head[u] * g.scale_head_ld + within[u]] = fine ? top / kMostE4m3 : NAN;
        }
    }
}

// ----------------------------------------------------------------------------------- reading ---

constexpr int kKeys = 32;                  // per step and wave
constexpr int kWaves = 4;
constexpr int kMaxSplits = 64;

// One product D += A B of a wave: A is 16 x 32, B is 32 x 16.  Lane l (quarter g = l / 16) holds row l % 16 of A and column l % 16 of B, eight
// neighbours 8 g .. 8 g + 7 of each, and of D column l % 16, rows 4 g .. 4 g + 3.
template <typename T> __device__ __forceinline__ f32x4 product16(s16x8 a, s16x8 b, f32x4 c);
template <> __device__ __forceinline__ f32x4 product16<__bf16>(s16x8 a, s16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 product16<_Float16>(s16x8 a, s16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <typename T> __device__ __forceinline__ s16x8 widened(uint2 v);
template <> __device__ __forceinline__ s16x8 widened<__bf16>(uint2 v)
{
    typedef __bf16 t2 __attribute__((ext_vector_type(2)));
    const t2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.x, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.x, 1.0f, true);
    const t2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.y, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.y, 1.0f, true);
    return __builtin_bit_cast(s16x8, bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]});
}
template <> __device__ __forceinline__ s16x8 widened<_Float16>(uint2 v)
{
    typedef _Float16 t2 __attribute__((ext_vector_type(2)));
    const t2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v.x, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v.x, 1.0f, true);
    const t2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v.y, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v.y, 1.0f, true);
    return __builtin_bit_cast(s16x8, f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]});
}

// A wave's tiles of 32 keys and values in LDS, as they lie in the cache, rows 16 bytes apart more than they are long: 4 r words modulo
// 64 banks are all different for sixteen rows, for both kinds of reads.  CHUNK: bytes of a load, 16 where all rows lie on 16.
template <int DP, int CHUNK>
struct Tiles8 {
    static constexpr int kPitch = DP + 16;
    static constexpr int kLanes = (DP == 64 ? 64 : 128) / CHUNK;           // per row of a load
    static constexpr int kPerPass = 64 / kLanes, kPasses = kKeys / kPerPass;
    static constexpr int kBytes = 2 * kKeys * kPitch + 3 * kKeys * 4;      // K, V; K's scales, V's, and their logarithms
    typedef unsigned Part __attribute__((ext_vector_type(CHUNK / 4)));
};

__device__ __forceinline__ long long shuffled(long long v, int from)
{
    const int lo = __shfl((int)v, from, 64), hi = __shfl((int)(v >> 32), from, 64);
    return (long long)((unsigned long long)(unsigned)lo | (unsigned long long)(unsigned)hi << 32);
}

// The larger, or the sum, of the four lanes of a column.
__device__ __forceinline__ float column_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return both_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float v) { return swapped_sum<32>(swapped_sum<16>(v)); }

// One block: ROWS rows (queries of the heads of one key head, see attention.h) as columns, sixteen to a tile; its keys in steps of 32 per wave,
// the four waves beside each other, each with its own tiles, maxima and sums, which are joined at the end.  Values stay in 8 bits up to the
// registers that feed the matrix units.  Scales of keys multiply the scores, those of values the weights before these are rounded.
//
// Bound by memory where a sequence has few rows: 32 tokens over histories of up to 16384 places, 32 heads over 8, dim 128 (695 MB) take 140 us (4.96
// TB/s, 5.2 in the kernel; a large copy reaches 4.9); vector units are busy for a quarter of the time, matrix units for 7 %.  With products
// of 32 columns, whose sums and queries take twice the registers (two waves per SIMD instead of three), 157 us; with two steps loaded
// ahead 158 at two waves, at three they do not fit.  A small call's 7 to 12 us are the waits from one lookup to the next: sequence, page, keys.
// Where a sequence has many rows every 32 of them load and widen its keys anew: 2048 new tokens over 16384 places, 32 heads over 8, dim 128, take 985
// us (0.52 PFLOP/s).
//
// All products are taken with the kept side as columns: S = K t(Q) leaves a lane the scores of keys 4 g .. and 16 + 4 g .. of its column, which,
// as weights, are the B operand of the next product as they lie; its A is the transposed tile of values, read in that order.
//
// Weights times scales are rounded to fp16 for the product with the values, whatever T is: it has three digits more than bf16, and holds e4m3
// exactly.  Its range: the maximum that a column's weights are taken against is that of score + log2(scale of the value), so that
// weights times scales lie where fp16 has most digits, whatever the scales are; the sum of the weights carries the same factor.  With
// weights in bf16, results of 32 tokens over 16384 places are 0.0023 off instead of 0.0017, which is what rounding them leaves.
template <typename T, int DP, int CHUNK, int ROWS>
__global__ void __launch_bounds__(256, ROWS == 16 ? 3 : 2) attention_cache_kernel(const CacheArgs a)
{
    using L = Tiles8<DP, CHUNK>;
    using W = _Float16;                                    // of the weights
    using lds_i32x2 = __attribute__((address_space(3))) i32x2;
    constexpr int NT = ROWS / 16, kSteps = DP / 32, kDims = DP / 16;
    constexpr int kJoinDims = 64 / NT, kJoinPitch = kJoinDims + 4;         // of all waves' sums at a time
    static_assert(kWaves * L::kBytes >= kWaves * ROWS * kJoinPitch * 4, "the joining takes the tiles' place");
    __shared__ __attribute__((aligned(256))) char lds[kWaves * L::kBytes];
    __shared__ float stats[kWaves][2][ROWS];

    const int kvh = blockIdx.x % a.kv_heads;
    const unsigned rest = blockIdx.x / a.kv_heads;
    const int split = rest % a.splits;
    const Work work = tile_at<false>(a, ROWS, rest / a.splits);
    if (!work.any)
        return;
    const Seq &x = work.x;
    const int first = work.first, rows = x.nq * a.group;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int before = (int)x.k0;                          // keys that are there already
    auto seen_by = [&](int place) { return a.causal && !a.tree ? min(max(place + before + 1, 0), x.nk) : x.nk; };
    const int seen_lo = a.tree ? min(max(before, 0), x.nk) : seen_by(quotient(a.by_group, first));

    int begin = 0, end = seen_by(quotient(a.by_group, min(first + ROWS, rows) - 1));
    if (a.splits > 1) {
        const int per = ((end + a.splits - 1) / a.splits + kKeys * kWaves - 1) / (kKeys * kWaves) * (kKeys * kWaves);
        begin = min(split * per, end);
        end = min(begin + per, end);
    }

    // what is loaded of a step: a row's place is that of lane % 32
    char *const kt = lds + wave * L::kBytes, *const vt = kt + kKeys * L::kPitch;
    float *const kscale = reinterpret_cast<float *>(vt + kKeys * L::kPitch), *const vscale = kscale + kKeys, *const vlog = vscale + kKeys;
    const Pages &pages = a.pages;
    const int *table = pages.table + work.seq * pages.table_ld;
    const int row = lane & 31, load_row = lane / L::kLanes, load_at = lane % L::kLanes * CHUNK;
    const bool loads = load_at < a.dim;
    const unsigned char *const kbase = pages.k + kvh * pages.head_ld + load_at, *const vbase = pages.v + kvh * pages.head_ld + load_at;
    const float *const sbase = (lane >= 32 ? pages.v_scale : pages.k_scale) + kvh * pages.scale_head_ld;
    typename L::Part kp[L::kPasses], vp[L::kPasses];
    float sc = 0.0f;
    auto page_at = [&](int j) { return min(max(table[quotient(pages.size, min(j + row, x.nk - 1))], 0), pages.count - 1); };
    auto load = [&](int j, int page) {
        const int key = min(j + row, x.nk - 1), within = key - quotient(pages.size, key) * (int)pages.size.d;
        const long long at = page * pages.page_ld + within * pages.place_ld;
        sc = sbase[page * pages.scale_page_ld + within];
#pragma unroll
        for (int i = 0; i < L::kPasses; ++i) {
            const long long from = shuffled(at, i * L::kPerPass + load_row);
            if (loads) {
                kp[i] = *reinterpret_cast<const typename L::Part *>(kbase + from);
                vp[i] = *reinterpret_cast<const typename L::Part *>(vbase + from);
            }
        }
    };
    constexpr int kStride = kKeys * kWaves;
    int j = begin + wave * kKeys, page = 0;
    if (j < end) {                                         // a step is loaded ahead, the pages of the one behind it too
        load(j, page_at(j));
        page = page_at(j + kStride);
    }

    int place[NT], seen[NT];
    float slope[NT];
    unsigned long long tree[NT];
    s16x8 q[NT][kSteps];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = first + n * 16 + col, at = min(r, rows - 1);
        place[n] = quotient(a.by_group, at);
        const int head = kvh * a.group + at - place[n] * a.group;
        seen[n] = seen_by(place[n]);
        tree[n] = a.tree ? (unsigned long long)a.tree[x.q0 + place[n]] : 0;
        slope[n] = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
        const T *from = row_of<const T>(a.q, x.q0 + place[n], head);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            q[n][i] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (r < rows && i * 32 + g * 8 < a.dim)
                q[n][i] = *reinterpret_cast<const s16x8 *>(from + i * 32 + g * 8);
        }
    }
    if (a.dim < DP) {                                      // zeros behind dim
        for (int i = lane * 16; i < 2 * kKeys * L::kPitch; i += 1024)
            *reinterpret_cast<uint4 *>(kt + i) = make_uint4(0, 0, 0, 0);
    }

    f32x4 o[NT][kDims];
    float m[NT], mc[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = -INFINITY, mc[n] = 0.0f, l[n] = 0.0f;
#pragma unroll
        for (int d = 0; d < kDims; ++d)
            o[n][d] = f32x4{};
    }
    const float c = a.cap > 0.0f ? 2.0f * kLog2e * a.scale / a.cap : a.scale * kLog2e, cap = a.cap * kLog2e;
    for (; j < end; j += kStride) {
        const bool masked = j + kKeys > seen_lo;
        // the tiles that were loaded, to LDS
        if (lane < 32) {
            kscale[row] = sc * c > 0x1.fffffep127f ? 0x1.fffffep127f : sc * c;     // (a score of 0 stays one; NaN stays NaN)
        } else {
            vscale[row] = sc;
            // (at least 2^-90, so that sums of weights stay within fp32's range; a scale that is not finite is no measure of the others: with an
            // infinite one as the maximum all weights, and their sum, would be 0)
            vlog[row] = __builtin_amdgcn_logf(sc < INFINITY ? fmaxf(sc, 0x1p-90f) : 0x1p-90f);
        }
        if (loads)
#pragma unroll
            for (int i = 0; i < L::kPasses; ++i) {
                const int to = i * L::kPerPass + load_row;
                *reinterpret_cast<typename L::Part *>(kt + to * L::kPitch + load_at) = kp[i];
                if (masked) {              // bytes that are no number would reach rows that do not see them: their row's scale says it instead
                    unsigned any = 0;
#pragma unroll
                    for (int u = 0; u < CHUNK / 4; ++u) {
                        const unsigned bad = ((vp[i][u] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                        vp[i][u] &= ~((bad >> 7) * 255u);
                        any |= bad;
                    }
                    if (any)
                        vscale[to] = NAN;
                }
                *reinterpret_cast<typename L::Part *>(vt + to * L::kPitch + load_at) = vp[i];
            }
        if (j + kStride < end) {
            load(j + kStride, page);
            page = page_at(j + 2 * kStride);
        }
        wave_sees();

        f32x4 p[NT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
                p[n][t] = f32x4{};
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const s16x8 k = widened<T>(*reinterpret_cast<const uint2 *>(kt + (t * 16 + col) * L::kPitch + i * 32 + g * 8));
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    p[n][t] = product16<T>(k, q[n][i], p[n][t]);
            }
        }
        f32x4 ks[2], vs[2], vl[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            ks[t] = *reinterpret_cast<const f32x4 *>(kscale + t * 16 + g * 4);
            vs[t] = *reinterpret_cast<const f32x4 *>(vscale + t * 16 + g * 4);
            vl[t] = *reinterpret_cast<const f32x4 *>(vlog + t * 16 + g * 4);
        }
        float top[NT];
        bool moves = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                p[n][t] *= ks[t];
            if (a.cap > 0.0f)
#pragma unroll
                for (int i = 0; i < 8; ++i)    // tanh(y) = 1 - 2 / (exp(2 y) + 1)
                    p[n][i / 4][i % 4] = fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(p[n][i / 4][i % 4]) + 1.0f), cap);
            if (a.slopes) {
                const float far = (float)(j + 4 * g - (place[n] + before));
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    p[n][i / 4][i % 4] = fmaf(-slope[n], fabsf(far + (float)(i / 4 * 16 + i % 4)), p[n][i / 4][i % 4]);
            }
            if (masked) {
                const int left = seen[n] - j - 4 * g, drafted = j + 4 * g - before;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int k = i / 4 * 16 + i % 4, bit = drafted + k;
                    bool sees = k < left;
                    if (a.tree && bit >= 0)
                        sees = sees && bit < 64 && (tree[n] >> (bit & 63) & 1);
                    if (!sees)
                        p[n][i / 4][i % 4] = -INFINITY;
                }
            }
            top[n] = p[n][0][0] + vl[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i)
                top[n] = fmaxf(top[n], p[n][i / 4][i % 4] + vl[i / 4][i % 4]);
            top[n] = column_max(top[n]);
            moves = moves || top[n] - m[n] > (float)kSlack<W>;
        }
        if (__any(moves)) {                                // see follow_max
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float next = fmaxf(m[n], top[n]), to = (next == -INFINITY ? 0.0f : next) - (float)kLift<W>;
                const float f = m[n] == -INFINITY ? 0.0f : exp2f(mc[n] - to);
                m[n] = next;
                mc[n] = to;
                l[n] *= f;
#pragma unroll
                for (int d = 0; d < kDims; ++d)
                    o[n][d] *= f;
            }
        }
        s16x8 b[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float weight = __builtin_amdgcn_exp2f(p[n][i / 4][i % 4] - mc[n]);
                l[n] += weight;
                w[i] = weight * vs[i / 4][i % 4];
                if (masked && p[n][i / 4][i % 4] == -INFINITY)
                    w[i] = 0.0f;           // (its scale may be no number)
            }
            b[n] = rounded<W>(w);
        }
        const int i8 = col >> 1, key = g * 4 + (i8 & 3) + (i8 >> 2) * 16;          // this lane's part of the transposing load
        const char *const from = vt + key * L::kPitch + (col & 1) * 8;
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            const auto v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(from + d * 16));
            const s16x8 w = widened<W>(make_uint2(v[0], v[1]));
#pragma unroll
            for (int n = 0; n < NT; ++n)
                o[n][d] = product16<W>(w, b[n], o[n][d]);
        }
        wave_sees();
    }

    // the four waves' sums
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] = column_sum(l[n]);
        if (g == 0) {
            stats[wave][0][n * 16 + col] = l[n] == 0.0f ? -INFINITY : m[n];        // (nothing seen: a sum of 0)
            stats[wave][1][n * 16 + col] = l[n];
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = n * 16 + col, r = first + at;
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i)
            top = fmaxf(top, stats[i][0][at]);
#pragma unroll
        for (int i = 0; i < kWaves; ++i)
            sum += stats[i][1][at] == 0.0f ? 0.0f : stats[i][1][at] * exp2f(stats[i][0][at] - top);
        const float mine = l[n] == 0.0f ? 0.0f : exp2f(m[n] - top);
        const float f = a.splits > 1 ? mine : sum > 0.0f ? mine / sum : sum == 0.0f ? 0.0f : NAN;
#pragma unroll
        for (int d = 0; d < kDims; ++d)
            o[n][d] *= f;
        if (r < rows && wave == 0 && g == 0) {
            const long long to = (x.q0 + place[n]) * a.heads + kvh * a.group + r - place[n] * a.group;
            if (a.splits > 1) {
                float *stat = a.parts + a.q_tokens * a.heads * a.splits * a.dim;
                stat[to * a.splits + split] = top;
                stat[(a.q_tokens * a.heads + to) * a.splits + split] = sum;
            } else if (a.lse) {
                a.lse[to] = sum == 0.0f ? -INFINITY : fmaf(top, 1.0f / kLog2e, log_of<W>(sum));
            }
        }
    }
    float *const join = reinterpret_cast<float *>(lds);
    const int jc = threadIdx.x / (kJoinDims / 4), jd = threadIdx.x % (kJoinDims / 4) * 4, jr = first + jc;
#pragma unroll
    for (int d0 = 0; d0 < DP; d0 += kJoinDims) {
        if (d0 >= a.dim)
            break;
        if (d0 > 0)
            __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int d = 0; d < kJoinDims / 16; ++d)
                if (d0 / 16 + d < kDims)
                    *reinterpret_cast<f32x4 *>(join + (wave * ROWS + n * 16 + col) * kJoinPitch + d * 16 + g * 4) = o[n][d0 / 16 + d < kDims ? d0 / 16 + d : 0];
        __syncthreads();
        if (jr >= rows || d0 + jd >= a.dim)
            continue;
        f32x4 v = *reinterpret_cast<const f32x4 *>(join + jc * kJoinPitch + jd);
#pragma unroll
        for (int i = 1; i < kWaves; ++i)
            v += *reinterpret_cast<const f32x4 *>(join + (i * ROWS + jc) * kJoinPitch + jd);
        const int jp = quotient(a.by_group, jr), jh = kvh * a.group + jr - jp * a.group;
        if (a.splits > 1) {
            *reinterpret_cast<f32x4 *>(a.parts + (((x.q0 + jp) * a.heads + jh) * a.splits + split) * a.dim + d0 + jd) = v;
        } else {
            typedef T t4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<t4 *>(row_of<T>(a.out, x.q0 + jp, jh) + d0 + jd) = t4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        }
    }
}

// Joins the splits of every row: a wave per row, whichever sequence it is of.  WIDE: a block per row, whose waves take eight splits each in turn (32
// rows of 48 splits: 10 us by waves, 5 by blocks).
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) attention_cache_join_kernel(const CacheArgs a)
{
    __shared__ float parts[4][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = WIDE ? (long long)blockIdx.x : (long long)blockIdx.x * 4 + wave, token = (unsigned)row / (unsigned)a.heads;
    if (token < offset_at(a.q_off, 0, a.off64) || token >= min(offset_at(a.q_off, a.seqs, a.off64), a.q_tokens))
        return;
    const int head = (int)(row - token * a.heads);
    const float *stat = a.parts + a.q_tokens * a.heads * a.splits * a.dim;
    const bool mine = lane < a.splits;
    const float m = mine ? stat[row * a.splits + lane] : -INFINITY, l = mine ? stat[(a.q_tokens * a.heads + row) * a.splits + lane] : 0.0f;
    float top = m;
#pragma unroll
    for (int i = 32; i > 0; i >>= 1)
        top = fmaxf(top, __shfl_xor(top, i, 64));
    const float w = l == 0.0f ? 0.0f : exp2f(m - top);
    const float sum = wave_sum(w * l);
    float o0 = 0.0f, o1 = 0.0f;
    const float *o = a.parts + row * a.splits * a.dim;
    const int d0 = min(lane, a.dim - 1), d1 = min(lane + 64, a.dim - 1);
    for (int i = WIDE ? wave * 8 : 0; i < a.splits; i += WIDE ? 32 : 8) {          // eight splits' loads in flight
        float v0[8], v1[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int k = min(i + u, a.splits - 1);
            v0[u] = o[(long long)k * a.dim + d0];
            v1[u] = o[(long long)k * a.dim + d1];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u < a.splits) {
                const float f = __shfl(w, i + u, 64);
                o0 = fmaf(f, v0[u], o0);
                o1 = fmaf(f, v1[u], o1);
            }
    }
    if (WIDE) {
        parts[wave][lane] = o0;
        parts[wave][lane + 64] = o1;
        __syncthreads();
        if (wave > 0)
            return;
        o0 = (parts[0][lane] + parts[1][lane]) + (parts[2][lane] + parts[3][lane]);
        o1 = (parts[0][lane + 64] + parts[1][lane + 64]) + (parts[2][lane + 64] + parts[3][lane + 64]);
    }
    const float f = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : NAN;
    T *out = row_of<T>(a.out, token, head);
    if (lane < a.dim)
        out[lane] = (T)(o0 * f);
    if (lane + 64 < a.dim)
        out[lane + 64] = (T)(o1 * f);
    if (a.lse && lane == 0)
        a.lse[row] = sum == 0.0f ? -INFINITY : fmaf(top, 1.0f / kLog2e, log_of<_Float16>(sum));
}

// -------------------------------------------------------------------------------------- host ---

int check_rows16(const char *what, const void *p, int64_t rows, int64_t token_ld, int64_t head_ld, int64_t heads, int64_t dim)
{
    if (!p)
        return rows > 0 ? report(FUSE_EINVAL, std::string(what) + " is NULL") : FUSE_OK;
    if (!on_16_bytes(p) || token_ld % 8 || head_ld % 8)
        return report(FUSE_EUNSUPPORTED, std::string(what) + ": rows are not on 16 bytes");
    if ((rows > 1 && token_ld < dim) || (heads > 1 && head_ld < dim))
        return report(FUSE_ESHAPE, std::string(what) + ": stride < dim");
    if (token_ld > (INT64_C(1) << 40) || head_ld > (INT64_C(1) << 40))
        return report(FUSE_EUNSUPPORTED, std::string(what) + ": stride > 2^40");
    return FUSE_OK;
}

int check_cache(const fuse_cache *f)
{
    if (!f)
        return report(FUSE_EINVAL, "cache is NULL");
    if (f->dtype != FUSE_BF16 && f->dtype != FUSE_F16)
        return report(known_dtype(f->dtype) ? FUSE_EUNSUPPORTED : FUSE_EINVAL, "dtype is neither FUSE_BF16 nor FUSE_F16");
    if (f->kv_heads < 1 || f->dim < 1 || f->tokens < 0 || f->seqs < 0 || f->pages < 0 || f->page_size < 1 || f->table_width < 0)
        return report(FUSE_EINVAL, "kv_heads, dim and page_size must be positive, counts must not be negative");
    if (f->dim % 8 || f->dim > kMaxDim)
        return report(FUSE_EUNSUPPORTED, "dim is no multiple of 8 up to " + std::to_string(kMaxDim));
    if (f->tokens >= (INT64_C(1) << 31) || f->pages >= (INT64_C(1) << 31) || f->seqs >= (1 << 24) || f->kv_heads > 4096 ||
        f->page_size > (1 << 30) || f->table_width >= (INT64_C(1) << 31))
        return report(FUSE_EUNSUPPORTED, "2^31 tokens, pages or pages of a sequence, 2^24 sequences, 4096 heads or 2^30 places per page, or more");
    if (f->table_width * f->page_size >= (INT64_C(1) << 31) - 4096)
        return report(FUSE_EUNSUPPORTED, "a sequence has room for 2^31 - 4096 places or more");
    if (f->seqs > 0 && f->tokens > 0) {
        if (!f->offsets || !f->lengths)
            return report(FUSE_EINVAL, "offsets or lengths is NULL");
        if (f->table_width > 0 && (!f->table || (f->seqs > 1 && f->table_ld < f->table_width)))
            return report(f->table ? FUSE_ESHAPE : FUSE_EINVAL, "table is NULL or its stride < table_width");
        if (f->pages > 0 && (!f->k || !f->v || !f->k_scale || !f->v_scale))
            return report(FUSE_EINVAL, "a part of the cache is NULL");
    }
    const uintptr_t width = f->offsets_are_64 ? 8 : 4;
    for (const void *p : {f->offsets, f->lengths})
        if (reinterpret_cast<uintptr_t>(p) % width)
            return report(FUSE_EINVAL, "offsets or lengths are not aligned to their type");
    for (const void *p : {(const void *)f->table, (const void *)f->k_scale, (const void *)f->v_scale})
        if (reinterpret_cast<uintptr_t>(p) % 4)
            return report(FUSE_EINVAL, "table or scales are not aligned to their type");
    for (const void *p : {f->k, f->v})
        if (reinterpret_cast<uintptr_t>(p) % 8)
            return report(FUSE_EUNSUPPORTED, "rows of the cache are not on 8 bytes");
    if (f->page_ld % 8 || f->head_ld % 8 || f->place_ld % 8)
        return report(FUSE_EUNSUPPORTED, "rows of the cache are not on 8 bytes");
    if ((f->page_size > 1 && f->place_ld < f->dim) || (f->kv_heads > 1 && f->head_ld < f->dim) || (f->pages > 1 && f->page_ld < f->dim) ||
        (f->kv_heads > 1 && f->scale_head_ld < 1) || (f->pages > 1 && f->scale_page_ld < 1))
        return report(FUSE_ESHAPE, "the cache's strides are less than its rows");
    for (int64_t ld : {f->page_ld, f->head_ld, f->place_ld, f->scale_page_ld, f->scale_head_ld, f->table_ld})
        if (ld > (INT64_C(1) << 40))
            return report(FUSE_EUNSUPPORTED, "stride > 2^40");
    return FUSE_OK;
}

CacheArgs cache_args(const fuse_cache *f)
{
    CacheArgs a = {};
    Pages &g = a.pages;
    g.k = static_cast<unsigned char *>(f->k), g.v = static_cast<unsigned char *>(f->v), g.k_scale = f->k_scale, g.v_scale = f->v_scale;
    g.page_ld = f->page_ld, g.head_ld = f->head_ld, g.place_ld = f->place_ld;
    g.scale_page_ld = f->scale_page_ld, g.scale_head_ld = f->scale_head_ld;
    g.table = f->table, g.table_ld = f->table_ld, g.count = (int)f->pages, g.width = f->pages > 0 ? (int)f->table_width : 0;
    g.size = divider((unsigned)f->page_size);
    a.q_off = f->offsets, a.lengths = f->lengths, a.off64 = f->offsets_are_64 != 0;
    a.q_tokens = f->tokens, a.seqs = (int)f->seqs, a.kv_heads = f->kv_heads, a.dim = f->dim, a.group = 1;
    return a;
}

int write_impl(const fuse_cache *f, const void *k, int64_t k_token_ld, int64_t k_head_ld, const void *v, int64_t v_token_ld, int64_t v_head_ld,
               void *stream)
{
    report(FUSE_OK, "");
    int rc = check_cache(f);
    if (!rc)
        rc = check_rows16("k", k, f->tokens, k_token_ld, k_head_ld, f->kv_heads, f->dim);
    if (!rc)
        rc = check_rows16("v", v, f->tokens, v_token_ld, v_head_ld, f->kv_heads, f->dim);
    if (rc)
        return rc;
    if (f->tokens == 0 || f->seqs == 0)
        return FUSE_OK;
    CacheArgs a = cache_args(f);
    a.k = {const_cast<void *>(k), k_token_ld, k_head_ld};
    a.v = {const_cast<void *>(v), v_token_ld, v_head_ld};
    a.by_row = divider(2 * (unsigned)f->kv_heads);
    const long long blocks = first_tile(f->tokens, (int)f->seqs, kWriteTokens);
    if (blocks >= 1 << 24)
        return report(FUSE_EUNSUPPORTED, "more tokens and sequences than one launch has blocks");
    if (f->dtype == FUSE_BF16)
        cache_write_kernel<__bf16><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(a);
    else
        cache_write_kernel<_Float16><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(a);
    return launched("cache_write_kernel");
}

// Rows of a block: sixteen where that is what a sequence has, on average.
int tile_of(const fuse_cache *f, const fuse_cache_query *q)
{
    return f->tokens * (q->heads / f->kv_heads) <= 16 * f->seqs ? 16 : 32;
}

long long tiles_of(const fuse_cache *f, const fuse_cache_query *q)
{
    return first_tile(f->tokens * (q->heads / f->kv_heads), (int)f->seqs, tile_of(f, q));
}

int check_read(const fuse_cache *f, const fuse_cache_query *q)
{
    int rc = check_cache(f);
    if (rc)
        return rc;
    if (!q)
        return report(FUSE_EINVAL, "query is NULL");
    if (q->heads < 1 || q->heads > 4096)
        return report(q->heads < 1 ? FUSE_EINVAL : FUSE_EUNSUPPORTED, "heads must lie between 1 and 4096");
    if (q->heads % f->kv_heads)
        return report(FUSE_ESHAPE, "heads is no multiple of kv_heads");
    if (!(q->scale >= 1e-30) || !(q->scale <= 1e30))
        return report(FUSE_EINVAL, "scale must lie between 1e-30 and 1e30");
    if (q->cap != 0.0 && (!(q->cap >= 1e-3) || !(q->cap <= 1e4)))
        return report(FUSE_EINVAL, "cap must be 0 (none) or lie between 1e-3 and 1e4 (capped scores are off by some 2^-22 of it)");
    if (q->tree && (!q->causal || q->slopes))
        return report(FUSE_EINVAL, "a tree goes with causal, and without slopes");
    if (reinterpret_cast<uintptr_t>(q->slopes) % 4 || reinterpret_cast<uintptr_t>(q->tree) % 8)
        return report(FUSE_EINVAL, "slopes or tree are not aligned to their type");
    if (f->tokens * q->heads >= (INT64_C(1) << 36) || tiles_of(f, q) * f->kv_heads >= (1 << 24))
        return report(FUSE_EUNSUPPORTED, "more tiles of queries than one launch has blocks");
    return check_rows16("q", q->q, f->tokens, q->q_token_ld, q->q_head_ld, q->heads, f->dim);
}

// Splits of the keys: as many as it takes to have three blocks for each of 256 compute units, of at least four steps of all waves each where
// all sequences fill their room (six blocks for 16 rows of dim 64, of which four fit at a time), or eight blocks of at least eight steps.  A split costs a
// block's beginning and end, some five steps, and the launch that joins them.  Calls from Python, one after the other:
//   eight steps, a goal of 512, 1024, 2048 and 4096 blocks: 32 tokens of 32 heads over 8, dim 128, over 16384 places each, filled to two thirds, take
//     151, 140, 143 and 149 us; 4 over 8192 places 21 with each;
//   four steps, a goal of 512, 768 and 1536: 16 tokens of these heads over 2048: 22.3, 21.6 and 21.7 us; 36 of 4 over 1 over 12168, filled to two thirds: 23.4,
//     22.8, 25.3; 8 of 64 over 8 of dim 80 over 8192: 25.1, 25.0, 29.4;
//   dim 64, four steps, 768 and 1536: 16 tokens of 8 heads over 4096: 21.6 and 20.5 us, of 16 over 8 22.2 and 21.2; 60 of 14 over 2 over 3000: 19.5 and 19.6; but
//     48 of 4 over 1 over 22826: 34.1 and 37.7.
// The room is the table's width; lengths are the device's.  Short sequences under wide tables have splits without keys, each of which ends, and is
// joined, like any other: 300 keys of a token of 32 heads over 8 take 11.7 us in a table of 320 places and 15.4 in one of 32768; 32 such tokens 11.4 and 18.9.
int splits_of(const fuse_cache *f, const fuse_cache_query *q)
{
    const long long blocks = std::max(1LL, tiles_of(f, q) * f->kv_heads), room = f->table_width * f->page_size, step = kKeys * kWaves;
    const long long goal = f->dim <= 64 && tile_of(f, q) == 16 ? 1536 : 768;
    const long long n = std::max(std::min(2048 / blocks, room / (8 * step)), std::min(goal / blocks, room / (4 * step)));
    return (int)std::max(1LL, std::min<long long>(n, kMaxSplits));
}

size_t read_bytes(const fuse_cache *f, const fuse_cache_query *q)
{
    const int splits = splits_of(f, q);
    return splits > 1 ? (size_t)f->tokens * q->heads * splits * (f->dim + 2) * sizeof(float) : 0;
}

template <typename T, int CHUNK, int ROWS>
void launch_dim(const CacheArgs &a, unsigned blocks, hipStream_t s)
{
    if (a.dim <= 64)
        attention_cache_kernel<T, 64, CHUNK, ROWS><<<blocks, 256, 0, s>>>(a);
    else if (a.dim <= 96)
        attention_cache_kernel<T, 96, CHUNK, ROWS><<<blocks, 256, 0, s>>>(a);
    else
        attention_cache_kernel<T, 128, CHUNK, ROWS><<<blocks, 256, 0, s>>>(a);
}

template <typename T>
int launch_read(const CacheArgs &a, unsigned tiles, hipStream_t s)
{
    const Pages &g = a.pages;
    const bool wide = a.dim % 16 == 0 && on_16_bytes(g.k) && on_16_bytes(g.v) && g.page_ld % 16 == 0 && g.head_ld % 16 == 0 && g.place_ld % 16 == 0;
    const unsigned blocks = tiles * a.kv_heads * a.splits;
    if (wide && a.tile == 16)
        launch_dim<T, 16, 16>(a, blocks, s);
    else if (wide)
        launch_dim<T, 16, 32>(a, blocks, s);
    else if (a.tile == 16)
        launch_dim<T, 8, 16>(a, blocks, s);
    else
        launch_dim<T, 8, 32>(a, blocks, s);
    int rc = launched("attention_cache_kernel");
    if (rc || a.splits == 1)
        return rc;
    const long long rows = a.q_tokens * a.heads;           // (fewer than 2^31: splits are for few rows)
    if (a.splits > 8)
        attention_cache_join_kernel<T, true><<<(unsigned)rows, 256, 0, s>>>(a);
    else
        attention_cache_join_kernel<T, false><<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(a);
    rc = launched("attention_cache_join_kernel");
    if (!rc)
        set_last_kernel("attention_cache_kernel");
    return rc;
}

int read_impl(const fuse_cache *f, const fuse_cache_query *q, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse, void *workspace,
              size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_read(f, q);
    if (!rc)
        rc = check_rows16("out", out, f->tokens, out_token_ld, out_head_ld, q->heads, f->dim);
    if (rc)
        return rc;
    if (reinterpret_cast<uintptr_t>(lse) % 4)
        return report(FUSE_EINVAL, "lse is not aligned to its type");
    if (f->tokens == 0 || f->seqs == 0)
        return FUSE_OK;
    const size_t need = read_bytes(f, q);
    if (need && (!workspace || !on_16_bytes(workspace) || workspace_bytes < need))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(need) + " bytes on 16 are needed");
    CacheArgs a = cache_args(f);
    a.q = {const_cast<void *>(q->q), q->q_token_ld, q->q_head_ld};
    a.out = {out, out_token_ld, out_head_ld};
    a.lse = lse, a.parts = static_cast<float *>(workspace);
    a.heads = q->heads, a.group = q->heads / f->kv_heads, a.by_group = divider((unsigned)a.group);
    a.causal = q->causal != 0, a.scale = (float)q->scale, a.cap = (float)q->cap, a.slopes = q->slopes;
    a.tree = reinterpret_cast<const long long *>(q->tree), a.splits = splits_of(f, q), a.tile = tile_of(f, q);
    const unsigned tiles = (unsigned)tiles_of(f, q);
    return f->dtype == FUSE_BF16 ? launch_read<__bf16>(a, tiles, (hipStream_t)stream) : launch_read<_Float16>(a, tiles, (hipStream_t)stream);
}

}  // namespace

extern "C" {

int fuse_cache_write(const fuse_cache *cache, const void *k, int64_t k_token_ld, int64_t k_head_ld, const void *v, int64_t v_token_ld,
                     int64_t v_head_ld, void *stream)
{
    return fuse::guard([&] { return write_impl(cache, k, k_token_ld, k_head_ld, v, v_token_ld, v_head_ld, stream); });
}

size_t fuse_attention_cache_bytes(const fuse_cache *cache, const fuse_cache_query *query)
{
    return fuse::guard_bytes([&] { return check_read(cache, query) ? 0 : read_bytes(cache, query); });
}

int fuse_attention_cache(const fuse_cache *cache, const fuse_cache_query *query, void *out, int64_t out_token_ld, int64_t out_head_ld, float *lse,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return read_impl(cache, query, out, out_token_ld, out_head_ld, lse, workspace, workspace_bytes, stream); });
}

}  // extern "C"
