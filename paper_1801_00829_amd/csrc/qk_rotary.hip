// Norms of queries and keys per head with the rotation by their positions (fuse_qk_rotary and its gradient).
//
//   n = x r w, r = 1 / sqrt(mean(x^2) + eps) over the dims of a head;  pair (a, b) of n:  a' = a cos - b sin,  b' = a sin + b cos
//   with angle = position * freq of the pair.
// Gradient, with g the gradient of the result turned back (by the negative angle) and gw = g o w:
//   dx = r (gw - x r^2 mean(gw o x)),  dw = sum over tokens and heads of g o x r
//
// Bound by memory: every row (a head of a token) is read once and written once.  A block takes some tokens at a time: first a table of
// their cos and sin, one pair per thread, which serves all heads; then the rows, several per wave.  A lane owns pairs, with both of a
// pair's dims, so that the rotation needs no other lane; it loads 16 bytes of each half (neighbours as pairs: 32 bytes in a row).
//
// 16384 tokens, 32 + 8 heads of dim 128, bf16: forward 71 us (4.7 TB/s; a large copy reaches 4.9), gradient 106 us with the 5 us that add up the
// weights' sums (4.8 TB/s, vector units busy for half of the time).  What the gradient took: the next row's loads ahead of this one's sums (132 ->
// 110 us; no gain forward: 71 and 73), sums over a wave by moves for many values at a time, without a branch for each (117 -> 108), 512
// persistent blocks instead of 1024 (109 -> 106, and 31 -> 24 for 5003 tokens of 16 heads of dim 80: 38 MB, where a block's beginning and
// end are what counts), all with as many turns (24 -> 22).
//
// Where a half of what turns, or of the rest, is no multiple of 16 bytes, or rows are not on them, all loads are of single elements: 16384 tokens, 32 + 8 heads of
// dim 96, bf16, with 24 dims turning take 126 us, gradients 291 (all dims turning: 50 and 94); 10628 tokens, 56 + 8 heads of dim 44, fp32, with 16
// turning 70 and 189 us (bytes alone: 49 and 73).
#include <algorithm>

#include "block_ops.h"

namespace {

using namespace fuse;

constexpr int kMaxDim = 256;
constexpr int kMaxPairs = kMaxDim / 2;
constexpr int kMaxAxes = 4;
constexpr int kTokens = 8;                 // per block at a time, at most
constexpr int kGradBlocks = 512;          // of a gradient call: each leaves one partial row of both weights' sums

struct Heads {                             // queries, or keys
    const void *x, *w;                     // w NULL: no norm
    const void *dy;                        // gradients: of the result
    void *out;                             // the result, or the gradient of x
    long long x_token, x_head, dy_token, dy_head, out_token, out_head;
    int heads;
    unsigned div_mul, div_shift;           // rows / heads, see token_of
};

struct RotaryArgs {
    Heads side[2];                         // queries, keys
    const void *positions;
    const double *freqs;
    double *partial_f64;                   // gradients: [2][blocks][dim] of the accumulators' type
    float *partial_f32;
    double eps;
    long long tokens, position_ld;
    int ends[kMaxAxes];                    // pairs of axis i and those before it
    int dim, half, neighbours, positions_are_64, per_turn;    // half: pairs that turn; per_turn: tokens of a block at a time
    int lanes;                             // of a row: a power of two
};

// r / heads for r < 2^31; exact, as the quotient is taken with 31 + n bits, 2^n the next power of two.
__device__ __forceinline__ int token_of(const Heads &h, int r)
{
    return h.heads == 1 ? r : (int)(__umulhi((unsigned)r, h.div_mul) >> h.div_shift);
}

// Sums of N values over aligned groups of `lanes` lanes, in all of them.
template <typename A, int N>
__device__ __forceinline__ void row_sums(A (&v)[N], int lanes)
{
#define FUSE_ALL(...)                                                                                                      \
    do {                                                                                                                  \
        _Pragma("unroll") for (int n = 0; n < N; ++n) __VA_ARGS__;                                                        \
    } while (0)
    if (lanes > 1)
        FUSE_ALL(v[n] += moved<0xB1>(v[n]));
    if (lanes > 2)
        FUSE_ALL(v[n] += moved<0x4E>(v[n]));
    if (lanes > 4)
        FUSE_ALL(v[n] += moved<0x141>(v[n]));
    if (lanes > 8)
        FUSE_ALL(v[n] += moved<0x140>(v[n]));
    if (lanes > 16)
        FUSE_ALL(v[n] = swapped_sum<16>(v[n]));
    if (lanes > 32)
        FUSE_ALL(v[n] = swapped_sum<32>(v[n]));
}

// Sums of N values over the lanes of a wave that are the same place of their groups, in all of them.
template <typename A, int N>
__device__ __forceinline__ void place_sums(A (&v)[N], int lanes)
{
    if (lanes <= 8)
        FUSE_ALL(v[n] += moved<0x128>(v[n]));              // eight lanes on within sixteen, then four, two, one
    if (lanes <= 4)
        FUSE_ALL(v[n] += moved<0x124>(v[n]));
    if (lanes <= 2)
        FUSE_ALL(v[n] += moved<0x122>(v[n]));
    if (lanes <= 1)
        FUSE_ALL(v[n] += moved<0x121>(v[n]));
    if (lanes <= 16)
        FUSE_ALL(v[n] = swapped_sum<16>(v[n]));
    if (lanes <= 32)
        FUSE_ALL(v[n] = swapped_sum<32>(v[n]));
}

template <typename A> struct Turn { A c, s; };

// cos and sin of an angle of 64 bits: whole turns are taken off in 64 bits, whatever the type.
__device__ __forceinline__ Turn<float> turn_of(double angle, float)
{
    double turns = angle * 0.15915494309189533577;     // 1 / (2 pi)
    turns -= rint(turns);
    Turn<float> t;
    sincospif((float)(2.0 * turns), &t.s, &t.c);
    return t;
}
__device__ __forceinline__ Turn<double> turn_of(double angle, double)
{
    Turn<double> t;
    sincos(angle, &t.s, &t.c);
    return t;
}

// The tokens' cos and sin, pair by pair; pairs behind those that turn get 1 and 0.
template <typename A>
__device__ __forceinline__ void fill_table(const RotaryArgs &a, Turn<A> *table, long long first, int tokens)
{
    const int pairs = a.dim / 2;
    for (int i = threadIdx.x; i < tokens * pairs; i += 256) {
        const int t = i / pairs, p = i - t * pairs;
        Turn<A> c = {(A)1, (A)0};
        if (p < a.half) {
            int axis = 0;
#pragma unroll
            for (int k = 0; k < kMaxAxes - 1; ++k)
                axis += p >= a.ends[k];
            const long long at = axis * a.position_ld + first + t;
            const double position = a.positions_are_64 ? (double)static_cast<const long long *>(a.positions)[at]
                                                       : (double)static_cast<const int *>(a.positions)[at];
            c = turn_of(position * a.freqs[p], (A)0);
        }
        table[i] = c;
    }
}

// A lane's pairs of a row, as they lie in memory: pair (k * lanes + l) * V + i for k < K, i < V.
template <typename T, int V> struct alignas(V * sizeof(T)) Pack { T t[V]; };

template <typename T, int V, int K, bool NEIGHBOURS>
struct Pairs {
    using A = typename acc_of<T>::type;
    Pack<T, V> u[K], v[K];

    __device__ __forceinline__ void load(const void *row, const int (&at)[K][2])
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at[k][0] >= 0) {
                u[k] = *reinterpret_cast<const Pack<T, V> *>(static_cast<const T *>(row) + at[k][0]);
                v[k] = *reinterpret_cast<const Pack<T, V> *>(static_cast<const T *>(row) + at[k][1]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    u[k].t[i] = v[k].t[i] = (T)0;
            }
    }
    __device__ __forceinline__ A first(int k, int i) const
    {
        return NEIGHBOURS && V > 1 ? (A)(2 * i < V ? u[k].t[2 * i % V] : v[k].t[2 * i % V]) : (A)u[k].t[i];
    }
    __device__ __forceinline__ A second(int k, int i) const
    {
        return NEIGHBOURS && V > 1 ? (A)(2 * i + 1 < V ? u[k].t[(2 * i + 1) % V] : v[k].t[(2 * i + 1) % V]) : (A)v[k].t[i];
    }
    __device__ __forceinline__ void set(int k, int i, A x, A y)
    {
        if (NEIGHBOURS && V > 1) {
            (2 * i < V ? u[k].t[2 * i % V] : v[k].t[2 * i % V]) = (T)x;
            (2 * i + 1 < V ? u[k].t[(2 * i + 1) % V] : v[k].t[(2 * i + 1) % V]) = (T)y;
        } else {
            u[k].t[i] = (T)x;
            v[k].t[i] = (T)y;
        }
    }
    __device__ __forceinline__ void store(void *row, const int (&at)[K][2]) const
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at[k][0] >= 0) {
                *reinterpret_cast<Pack<T, V> *>(static_cast<T *>(row) + at[k][0]) = u[k];
                *reinterpret_cast<Pack<T, V> *>(static_cast<T *>(row) + at[k][1]) = v[k];
            }
    }
};

// Where a lane's pairs lie in a row; -1: behind the last one.
template <int V, int K, bool NEIGHBOURS>
__device__ __forceinline__ void places(const RotaryArgs &a, int lane, int (&at)[K][2])
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int p = (k * a.lanes + lane) * V;
        if (p >= a.dim / 2)
            at[k][0] = at[k][1] = -1;
        else if (NEIGHBOURS) {
            at[k][0] = 2 * p;
            at[k][1] = 2 * p + (V > 1 ? V : 1);
        } else {                           // halves of what turns, then halves of the rest
            at[k][0] = p < a.half ? p : p + a.half;
            at[k][1] = p < a.half ? p + a.half : p + a.dim / 2;
        }
    }
}

template <typename T>
__device__ __forceinline__ T *row_at(const void *p, long long token, int head, long long token_ld, long long head_ld)
{
    return static_cast<T *>(const_cast<void *>(p)) + token * token_ld + head * head_ld;
}

// For all of a lane's pairs.
#define FUSE_PAIRS(...)                                                                                                    \
    do {                                                                                                                  \
        _Pragma("unroll") for (int k = 0; k < K; ++k) _Pragma("unroll") for (int i = 0; i < V; ++i) { __VA_ARGS__; }      \
    } while (0)

template <typename T, int V, int K, bool NEIGHBOURS>
__global__ void __launch_bounds__(256) qk_rotary_kernel(const RotaryArgs a)
{
    using A = typename acc_of<T>::type;
    using P = Pairs<T, V, K, NEIGHBOURS>;
    __shared__ Turn<A> table[kTokens * kMaxPairs];
    const int lane = threadIdx.x & (a.lanes - 1), mine = threadIdx.x / a.lanes, step = 256 / a.lanes, pairs = a.dim / 2;
    int at[K][2];
    places<V, K, NEIGHBOURS>(a, lane, at);
    for (long long first = (long long)blockIdx.x * a.per_turn; first < a.tokens; first += (long long)gridDim.x * a.per_turn) {
        const int tokens = (int)min((long long)a.per_turn, a.tokens - first);
        fill_table<A>(a, table, first, tokens);
        __syncthreads();
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const Heads &h = a.side[side];
            const int rows = tokens * h.heads;
            P w;
            if (h.w)
                w.load(h.w, at);
            for (int r = mine; r < rows; r += step) {
                const int t = token_of(h, r), head = r - t * h.heads;
                P x;
                x.load(row_at<const T>(h.x, first + t, head, h.x_token, h.x_head), at);
                A scale = (A)1;
                if (h.w) {
                    A sum[1] = {(A)0};
                    FUSE_PAIRS(sum[0] += x.first(k, i) * x.first(k, i) + x.second(k, i) * x.second(k, i));
                    row_sums(sum, a.lanes);
                    scale = (A)1 / sqrt(sum[0] / (A)a.dim + (A)a.eps);
                }
                const Turn<A> *turn = table + t * pairs;
                FUSE_PAIRS(
                    A u = x.first(k, i); A v = x.second(k, i);
                    if (h.w) {
                        u *= scale * w.first(k, i);
                        v *= scale * w.second(k, i);
                    }
                    const Turn<A> c = turn[min((k * a.lanes + lane) * V, pairs - V) + i];
                    x.set(k, i, u * c.c - v * c.s, u * c.s + v * c.c));
                x.store(row_at<T>(h.out, first + t, head, h.out_token, h.out_head), at);
            }
        }
        __syncthreads();
    }
}

template <typename T, int V, int K, bool NEIGHBOURS>
__global__ void __launch_bounds__(256) qk_rotary_grad_kernel(const RotaryArgs a)
{
    using A = typename acc_of<T>::type;
    using P = Pairs<T, V, K, NEIGHBOURS>;
    __shared__ Turn<A> table[kTokens * kMaxPairs];
    __shared__ A sums[2][4][kMaxDim];
    const int lane = threadIdx.x & (a.lanes - 1), mine = threadIdx.x / a.lanes, step = 256 / a.lanes, pairs = a.dim / 2;
    int at[K][2];
    places<V, K, NEIGHBOURS>(a, lane, at);
    A dw[2][2 * K * V] = {};
    for (long long first = (long long)blockIdx.x * a.per_turn; first < a.tokens; first += (long long)gridDim.x * a.per_turn) {
        const int tokens = (int)min((long long)a.per_turn, a.tokens - first);
        auto load = [&](const Heads &h, int r, P &x, P &g) {
            if (r < tokens * h.heads) {
                const int t = token_of(h, r), head = r - t * h.heads;
                g.load(row_at<const T>(h.dy, first + t, head, h.dy_token, h.dy_head), at);
                if (h.w)
                    x.load(row_at<const T>(h.x, first + t, head, h.x_token, h.x_head), at);
            }
        };
        P ahead_x[2], ahead_g[2];          // the first rows of both are asked for before the table is made
        load(a.side[0], mine, ahead_x[0], ahead_g[0]);
        load(a.side[1], mine, ahead_x[1], ahead_g[1]);
        fill_table<A>(a, table, first, tokens);
        __syncthreads();
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const Heads &h = a.side[side];
            const int rows = tokens * h.heads;
            P w;
            if (h.w)
                w.load(h.w, at);
            for (int r = mine; r < rows; r += step) {
                const int t = token_of(h, r), head = r - t * h.heads;
                P x = ahead_x[side], g = ahead_g[side];
                load(h, r + step, ahead_x[side], ahead_g[side]);
                const Turn<A> *turn = table + t * pairs;
                A gu[K][V], gv[K][V];      // turned back
                FUSE_PAIRS(
                    const Turn<A> c = turn[min((k * a.lanes + lane) * V, pairs - V) + i];
                    gu[k][i] = g.first(k, i) * c.c + g.second(k, i) * c.s;
                    gv[k][i] = g.second(k, i) * c.c - g.first(k, i) * c.s);
                if (h.w) {
                    A sum[2] = {(A)0, (A)0};               // of squares, and of the products with the gradient
                    FUSE_PAIRS(
                        sum[0] += x.first(k, i) * x.first(k, i) + x.second(k, i) * x.second(k, i);
                        sum[1] += gu[k][i] * w.first(k, i) * x.first(k, i) + gv[k][i] * w.second(k, i) * x.second(k, i));
                    row_sums(sum, a.lanes);
                    const A scale = (A)1 / sqrt(sum[0] / (A)a.dim + (A)a.eps);
                    const A mean = sum[1] / (A)a.dim * scale * scale;
                    FUSE_PAIRS(
                        dw[side][2 * (k * V + i)] += gu[k][i] * (x.first(k, i) * scale);
                        dw[side][2 * (k * V + i) + 1] += gv[k][i] * (x.second(k, i) * scale);
                        gu[k][i] = scale * (gu[k][i] * w.first(k, i) - x.first(k, i) * mean);
                        gv[k][i] = scale * (gv[k][i] * w.second(k, i) - x.second(k, i) * mean));
                }
                FUSE_PAIRS(g.set(k, i, gu[k][i], gv[k][i]));
                g.store(row_at<T>(h.out, first + t, head, h.out_token, h.out_head), at);
            }
        }
        __syncthreads();
    }
    // the weights' sums of this block: over the rows of a wave, then over its waves
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        if (!a.side[side].w)
            continue;
        place_sums(dw[side], a.lanes);
        if ((threadIdx.x & 63) < a.lanes)
            FUSE_PAIRS(
                if (at[k][0] >= 0) {
                    sums[side][wave][at[k][0] + (NEIGHBOURS && V > 1 ? 2 * i : i)] = dw[side][2 * (k * V + i)];
                    sums[side][wave][NEIGHBOURS && V > 1 ? at[k][0] + 2 * i + 1 : at[k][1] + i] = dw[side][2 * (k * V + i) + 1];
                });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.dim; i += 256) {
        const int side = i >= a.dim, c = i - side * a.dim;
        if (!a.side[side].w)
            continue;
        const A s = (sums[side][0][c] + sums[side][1][c]) + (sums[side][2][c] + sums[side][3][c]);
        const long long to = ((long long)side * gridDim.x + blockIdx.x) * a.dim + c;
        if constexpr (sizeof(A) == 8)
            a.partial_f64[to] = s;
        else
            a.partial_f32[to] = s;
    }
}

// The weights' gradients from the blocks' partial rows, in order: 16 columns of one weight per block, 64 slices of the partial rows.
template <typename T>
__global__ void __launch_bounds__(1024) qk_rotary_sums_kernel(const void *partial, int blocks, int dim, T *dq_weight, T *dk_weight)
{
    using A = typename acc_of<T>::type;
    __shared__ A part[64][17];
    T *out = blockIdx.y ? dk_weight : dq_weight;
    if (!out)
        return;
    const int col = threadIdx.x & 15, c = blockIdx.x * 16 + col, slice = threadIdx.x >> 4;
    const A *p = static_cast<const A *>(partial) + (long long)blockIdx.y * blocks * dim;
    A s = (A)0;
    if (c < dim)
#pragma unroll 8
        for (int b = slice; b < blocks; b += 64)
            s += p[(long long)b * dim + c];
    part[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < dim) {
#pragma unroll 16
        for (int i = 1; i < 64; ++i)
            s += part[i][col];
        out[c] = (T)s;
    }
}

// ------------------------------------------------------------------------------------ host ---

int check_side(const fuse_rotary *f, const void *p, int64_t token_ld, int64_t head_ld, int64_t heads, const char *what)
{
    if (!p)
        return f->tokens > 0 ? report(FUSE_EINVAL, std::string(what) + " is NULL") : FUSE_OK;
    if (reinterpret_cast<uintptr_t>(p) % dtype_size(f->dtype))
        return report(FUSE_EINVAL, std::string(what) + " is not aligned to its type");
    if ((f->tokens > 1 && token_ld < f->dim) || (heads > 1 && head_ld < f->dim))
        return report(FUSE_ESHAPE, std::string(what) + ": stride < dim");
    if (token_ld > (INT64_C(1) << 40) || head_ld > (INT64_C(1) << 40))
        return report(FUSE_EUNSUPPORTED, std::string(what) + ": stride > 2^40");
    return FUSE_OK;
}

int check_rotary(const fuse_rotary *f)
{
    if (!f)
        return report(FUSE_EINVAL, "rotary is NULL");
    if (!known_dtype(f->dtype))
        return report(FUSE_EINVAL, "dtype is not a fuse_dtype");
    if (f->pairs != FUSE_PAIR_HALVES && f->pairs != FUSE_PAIR_NEIGHBOURS)
        return report(FUSE_EINVAL, "pairs is not a fuse_pair_kind");
    if (f->heads < 1 || f->kv_heads < 0 || f->dim < 1 || f->tokens < 0)
        return report(FUSE_EINVAL, "heads and dim must be positive, kv_heads and tokens must not be negative");
    if (f->dim % 2 || f->dim > kMaxDim)
        return report(FUSE_EUNSUPPORTED, "dim is no multiple of 2 up to " + std::to_string(kMaxDim));
    if (f->heads > 4096 || f->kv_heads > 4096 || f->tokens >= (INT64_C(1) << 31))
        return report(FUSE_EUNSUPPORTED, "4096 heads or 2^31 tokens, or more");
    if (f->axes < 1 || f->axes > kMaxAxes)
        return report(FUSE_EINVAL, "axes must lie between 1 and " + std::to_string(kMaxAxes));
    int64_t half = 0;
    for (int i = 0; i < f->axes; ++i) {
        if (f->sections[i] < 0)
            return report(FUSE_EINVAL, "sections must not be negative");
        half += f->sections[i];
    }
    if (half < 1 || 2 * half > f->dim)
        return report(FUSE_ESHAPE, "sections have " + std::to_string(half) + " pairs, a head has " + std::to_string(f->dim / 2));
    if (!(f->eps >= 0.0))
        return report(FUSE_EINVAL, "eps must not be negative");
    if (f->kv_heads == 0 && f->k_weight)
        return report(FUSE_EINVAL, "k_weight needs keys");
    if (f->tokens > 0 && (!f->positions || !f->freqs))
        return report(FUSE_EINVAL, "positions or freqs is NULL");
    if (reinterpret_cast<uintptr_t>(f->positions) % (f->positions_are_64 ? 8 : 4) || reinterpret_cast<uintptr_t>(f->freqs) % 8)
        return report(FUSE_EINVAL, "positions or freqs are not aligned to their type");
    if (f->axes > 1 && f->position_ld != 0 && (f->position_ld < f->tokens || f->position_ld > (INT64_C(1) << 40)))
        return report(FUSE_ESHAPE, "position_ld is neither 0 nor as many as tokens");
    for (const void *p : {f->q_weight, f->k_weight})
        if (reinterpret_cast<uintptr_t>(p) % dtype_size(f->dtype))
            return report(FUSE_EINVAL, "a weight is not aligned to its type");
    return FUSE_OK;
}

RotaryArgs rotary_args(const fuse_rotary *f)
{
    RotaryArgs a = {};
    a.positions = f->positions, a.freqs = f->freqs, a.eps = f->eps, a.tokens = f->tokens, a.position_ld = f->axes > 1 ? f->position_ld : 0;
    int end = 0;
    for (int i = 0; i < kMaxAxes; ++i)
        a.ends[i] = end += i < f->axes ? f->sections[i] : 0;
    a.half = end, a.dim = f->dim, a.neighbours = f->pairs == FUSE_PAIR_NEIGHBOURS, a.positions_are_64 = f->positions_are_64 != 0;
    for (int i = f->axes - 1; i < kMaxAxes; ++i)
        a.ends[i] = a.half;                // (pairs that turn are before the last axis's end)
    a.side[0].x = f->q, a.side[0].w = f->q_weight, a.side[0].x_token = f->q_token_ld, a.side[0].x_head = f->q_head_ld, a.side[0].heads = f->heads;
    a.side[1].x = f->k, a.side[1].w = f->k_weight, a.side[1].x_token = f->k_token_ld, a.side[1].x_head = f->k_head_ld;
    a.side[1].heads = f->kv_heads;
    for (Heads &h : a.side) {
        int n = 0;
        while ((1 << n) < h.heads)
            ++n;
        h.div_mul = h.heads > 0 ? (unsigned)(((unsigned long long)1 << (31 + n)) / (unsigned)h.heads + 1) : 0;
        h.div_shift = n > 0 ? n - 1 : 0;
    }
    return a;
}

bool on_16(const fuse_rotary *f, const void *p, int64_t token_ld, int64_t head_ld, int64_t heads)
{
    const int64_t per = 16 / (int64_t)dtype_size(f->dtype);
    return !p || (on_16_bytes(p) && (f->tokens <= 1 || token_ld % per == 0) && (heads <= 1 || head_ld % per == 0));
}

// Whether a lane's pairs can be loaded 16 bytes at a time: every row on 16 bytes, and each half of a multiple of those.
bool wide(const fuse_rotary *f, const RotaryArgs &a)
{
    const int v = 16 / (int)dtype_size(f->dtype);
    if (a.neighbours ? a.dim / 2 % v : a.half % v || (a.dim / 2 - a.half) % v)
        return false;
    for (const Heads &h : a.side)
        if (!on_16(f, h.x, h.x_token, h.x_head, h.heads) || !on_16(f, h.dy, h.dy_token, h.dy_head, h.heads) ||
            !on_16(f, h.out, h.out_token, h.out_head, h.heads) || !on_16_bytes(h.w))
            return false;
    return true;
}

// Lanes per row: as many as its pairs take, a power of two, 64 at most.
int lanes_for(int pairs, int v)
{
    int n = 1;
    while (n < 64 && n * v < pairs)
        n *= 2;
    return n;
}

int64_t turns(const RotaryArgs &a) { return (a.tokens + a.per_turn - 1) / a.per_turn; }

template <typename T, bool GRAD, int V, int K, bool NEIGHBOURS>
void launch(const RotaryArgs &a, unsigned blocks, hipStream_t s)
{
    if (GRAD)
        qk_rotary_grad_kernel<T, V, K, NEIGHBOURS><<<blocks, 256, 0, s>>>(a);
    else
        qk_rotary_kernel<T, V, K, NEIGHBOURS><<<blocks, 256, 0, s>>>(a);
}

template <typename T, bool GRAD>
void launch_type(RotaryArgs a, bool vec, unsigned blocks, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    a.lanes = lanes_for(a.dim / 2, vec ? V : 1);
    if (vec && a.neighbours)
        launch<T, GRAD, V, 1, true>(a, blocks, s);
    else if (vec)
        launch<T, GRAD, V, 1, false>(a, blocks, s);
    else if (a.dim / 2 <= 64 && a.neighbours)
        launch<T, GRAD, 1, 1, true>(a, blocks, s);
    else if (a.dim / 2 <= 64)
        launch<T, GRAD, 1, 1, false>(a, blocks, s);
    else if (a.neighbours)
        launch<T, GRAD, 1, 2, true>(a, blocks, s);
    else
        launch<T, GRAD, 1, 2, false>(a, blocks, s);
}

template <bool GRAD>
void launch_any(int dtype, const RotaryArgs &a, bool vec, unsigned blocks, hipStream_t s)
{
    switch (dtype) {
    case FUSE_F64: launch_type<double, GRAD>(a, vec, blocks, s); break;
    case FUSE_F32: launch_type<float, GRAD>(a, vec, blocks, s); break;
    case FUSE_BF16: launch_type<__bf16, GRAD>(a, vec, blocks, s); break;
    default: launch_type<_Float16, GRAD>(a, vec, blocks, s); break;
    }
}

// Tokens of a block at a time: as many as it takes for the keys' rows to fill a block's lanes, but no more than leave 512 blocks, all with as
// many turns.
int per_turn_for(const fuse_rotary *f)
{
    const int rows = 256 / lanes_for(f->dim / 2, 16 / (int)dtype_size(f->dtype)), heads = f->kv_heads > 0 ? std::min(f->heads, f->kv_heads) : f->heads;
    const int64_t most = std::min((rows + heads - 1) / heads, kTokens);
    const int64_t each = std::max<int64_t>(1, (f->tokens + kGradBlocks * most - 1) / (kGradBlocks * most));
    return (int)std::max<int64_t>(1, (f->tokens + kGradBlocks * each - 1) / (kGradBlocks * each));
}

int rotary_impl(const fuse_rotary *f, void *q_out, int64_t q_token_ld, int64_t q_head_ld, void *k_out, int64_t k_token_ld, int64_t k_head_ld,
                void *stream)
{
    report(FUSE_OK, "");
    int rc = check_rotary(f);
    if (rc)
        return rc;
    if ((rc = check_side(f, f->q, f->q_token_ld, f->q_head_ld, f->heads, "q")) ||
        (rc = check_side(f, q_out, q_token_ld, q_head_ld, f->heads, "q_out")))
        return rc;
    if (f->kv_heads > 0 && ((rc = check_side(f, f->k, f->k_token_ld, f->k_head_ld, f->kv_heads, "k")) ||
                            (rc = check_side(f, k_out, k_token_ld, k_head_ld, f->kv_heads, "k_out"))))
        return rc;
    if (f->tokens == 0)
        return FUSE_OK;
    RotaryArgs a = rotary_args(f);
    a.side[0].out = q_out, a.side[0].out_token = q_token_ld, a.side[0].out_head = q_head_ld;
    a.side[1].out = k_out, a.side[1].out_token = k_token_ld, a.side[1].out_head = k_head_ld;
    a.per_turn = per_turn_for(f);
    launch_any<false>(f->dtype, a, wide(f, a), (unsigned)std::min<int64_t>(turns(a), 16384), (hipStream_t)stream);
    return launched("qk_rotary_kernel");
}

int grad_blocks(const fuse_rotary *f)
{
    const int64_t per = per_turn_for(f), turns = (f->tokens + per - 1) / per, each = (turns + kGradBlocks - 1) / kGradBlocks;
    return each ? (int)((turns + each - 1) / each) : 0;    // (all blocks with as many turns)
}

size_t grad_bytes(const fuse_rotary *f) { return (size_t)2 * grad_blocks(f) * f->dim * (f->dtype == FUSE_F64 ? 8 : 4); }

template <typename T>
void launch_sums(const void *partial, int blocks, int dim, void *dq_weight, void *dk_weight, hipStream_t s)
{
    qk_rotary_sums_kernel<T><<<dim3((dim + 15) / 16, 2), 1024, 0, s>>>(partial, blocks, dim, static_cast<T *>(dq_weight), static_cast<T *>(dk_weight));
}

int rotary_grad_impl(const fuse_rotary *f, const fuse_rotary_grads *g, void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_rotary(f);
    if (rc)
        return rc;
    if (!g)
        return report(FUSE_EINVAL, "grads is NULL");
    if ((rc = check_side(f, g->dq_out, g->dq_out_token_ld, g->dq_out_head_ld, f->heads, "dq_out")) ||
        (rc = check_side(f, g->dq, g->dq_token_ld, g->dq_head_ld, f->heads, "dq")) ||
        (rc = f->q_weight ? check_side(f, f->q, f->q_token_ld, f->q_head_ld, f->heads, "q") : FUSE_OK))
        return rc;
    if (f->kv_heads > 0 && ((rc = check_side(f, g->dk_out, g->dk_out_token_ld, g->dk_out_head_ld, f->kv_heads, "dk_out")) ||
                            (rc = check_side(f, g->dk, g->dk_token_ld, g->dk_head_ld, f->kv_heads, "dk")) ||
                            (rc = f->k_weight ? check_side(f, f->k, f->k_token_ld, f->k_head_ld, f->kv_heads, "k") : FUSE_OK)))
        return rc;
    if ((!g->dq_weight) != (!f->q_weight) || (!g->dk_weight) != (!f->k_weight))
        return report(FUSE_EINVAL, "dq_weight and dk_weight go with q_weight and k_weight");
    for (const void *p : {g->dq_weight, g->dk_weight})
        if (reinterpret_cast<uintptr_t>(p) % dtype_size(f->dtype))
            return report(FUSE_EINVAL, "a weight's gradient is not aligned to its type");
    const bool sums = f->q_weight || f->k_weight;
    if (sums && f->tokens > 0 && (!workspace || !on_16_bytes(workspace) || workspace_bytes < grad_bytes(f)))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(grad_bytes(f)) + " bytes on 16 are needed");
    RotaryArgs a = rotary_args(f);
    a.side[0].dy = g->dq_out, a.side[0].dy_token = g->dq_out_token_ld, a.side[0].dy_head = g->dq_out_head_ld;
    a.side[0].out = g->dq, a.side[0].out_token = g->dq_token_ld, a.side[0].out_head = g->dq_head_ld;
    a.side[1].dy = g->dk_out, a.side[1].dy_token = g->dk_out_token_ld, a.side[1].dy_head = g->dk_out_head_ld;
    a.side[1].out = g->dk, a.side[1].out_token = g->dk_token_ld, a.side[1].out_head = g->dk_head_ld;
    for (Heads &h : a.side)
        if (!h.w)
            h.x = nullptr;                 // not read
    a.partial_f32 = static_cast<float *>(workspace);
    a.partial_f64 = static_cast<double *>(workspace);
    a.per_turn = per_turn_for(f);
    const int blocks = grad_blocks(f);
    if (f->tokens > 0) {
        launch_any<true>(f->dtype, a, wide(f, a), (unsigned)blocks, (hipStream_t)stream);
        if ((rc = launched("qk_rotary_grad_kernel")))
            return rc;
    }
    if (!sums)
        return FUSE_OK;
    // (without tokens the sums are those of nothing: zeros)
    switch (f->dtype) {
    case FUSE_F64: launch_sums<double>(workspace, blocks, f->dim, g->dq_weight, g->dk_weight, (hipStream_t)stream); break;
    case FUSE_F32: launch_sums<float>(workspace, blocks, f->dim, g->dq_weight, g->dk_weight, (hipStream_t)stream); break;
    case FUSE_BF16: launch_sums<__bf16>(workspace, blocks, f->dim, g->dq_weight, g->dk_weight, (hipStream_t)stream); break;
    default: launch_sums<_Float16>(workspace, blocks, f->dim, g->dq_weight, g->dk_weight, (hipStream_t)stream); break;
    }
    rc = launched("qk_rotary_sums_kernel");
    if (!rc && f->tokens > 0)
        set_last_kernel("qk_rotary_grad_kernel");
    return rc;
}

}  // namespace

extern "C" {

int fuse_qk_rotary(const fuse_rotary *rotary, void *q_out, int64_t q_token_ld, int64_t q_head_ld, void *k_out, int64_t k_token_ld,
                   int64_t k_head_ld, void *stream)
{
    return fuse::guard([&] { return rotary_impl(rotary, q_out, q_token_ld, q_head_ld, k_out, k_token_ld, k_head_ld, stream); });
}

size_t fuse_qk_rotary_backward_bytes(const fuse_rotary *rotary)
{
    return fuse::guard_bytes([&] { return check_rotary(rotary) || (!rotary->q_weight && !rotary->k_weight) ? 0 : grad_bytes(rotary); });
}

int fuse_qk_rotary_backward(const fuse_rotary *rotary, const fuse_rotary_grads *grads, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return rotary_grad_impl(rotary, grads, workspace, workspace_bytes, stream); });
}

}  // extern "C"
