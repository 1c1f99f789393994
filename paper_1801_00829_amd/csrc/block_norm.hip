// Norms before and after a block, fused with the block's gate and its residual scale (fuse_block_norm and its gradient).
//
//   u = N_post(z) or z;   h = x + scale * gate o u;   y = N_pre(h)
//   N(v) = v r w, r = 1 / sqrt(mean(v^2) + eps)                        (rms)
//   N(v) = (v - m) r w + b, r = 1 / sqrt(mean((v - m)^2) + eps)        (layer)
//
// Gradient, with n = v r (or (v - m) r) the normalised row, g = dy o w:
//   dv = r (g - n mean(g n) [- mean(g)]),  dw = sum over the rows of dy o n,  db = sum over the rows of dy
//   dx = dh + dv(h);  dgate = scale dx o u, summed over what the gate is broadcast over;  dz = dv(z) of scale dx o gate
//
// Bound by memory: a row is read once and stays in registers through all its statistics.  A group of G threads owns a row,
// eight columns per thread and step, so a row of up to 8192 columns is one step; up to 32768 columns are four.  Statistics
// of a layer norm are taken in two passes over the registers (mean, then squares of the differences): one pass of sums of
// squares would lose the digits that a large mean has.
#include "block_ops.h"

namespace {

using namespace fuse;

constexpr int V = 8;                       // columns per thread and step
constexpr int kMaxCols = 32768;            // 1024 threads x 4 steps
constexpr int kMaxThreads = 1024;
constexpr int kGradBlocks = 512;           // blocks of a gradient call: each leaves one partial row of every column sum

struct Gate {
    int kind;                              // 0: none, 1: per column, 2: per row, 3: per cell
    const void *p;
    long long ld;
};

struct FwdArgs {
    const void *x, *z, *post_w, *post_b, *pre_w, *pre_b;
    void *h, *y;
    long long x_ld, z_ld, h_ld, y_ld, rows;
    int cols, group;                       // group: threads per row
    Gate gate;
    double eps, scale;
};

struct BwdArgs {
    const void *dh, *dy, *h, *z, *post_w, *post_b, *pre_w;
    void *dx, *dz, *dgate, *partial;       // partial: [5][blocks][cols]
    long long dh_ld, dy_ld, h_ld, z_ld, dx_ld, dz_ld, dgate_ld, rows;
    int cols, group;
    Gate gate;
    double eps, scale;
    int want_dpre_w, want_dpre_b, want_dpost_w, want_dpost_b;
};

struct SumArgs {
    const void *partial;                   // [5][blocks][cols]
    void *out[5];                          // NULL: not asked for
    int blocks, cols;
};

// Column of element j of a thread's step k.  VEC: eight neighbours, loaded 16 bytes at a time (every row and pointer on
// 16 bytes, columns a multiple of 8).  Else neighbouring threads take neighbouring columns, so that loads of single
// elements still cover whole cache lines.
template <bool VEC>
__device__ __forceinline__ int col_of(int k, int j, int lane, int group)
{
    return VEC ? (k * group + lane) * V + j : (k * V + j) * group + lane;
}

// A thread's part of a row as it lies in memory: what is loaded ahead of its use stays in the row's own type.
template <typename T, int K>
struct Part {
    struct alignas(16) Pack { T t[16 / sizeof(T)]; };
    static constexpr int N = 16 / sizeof(T);
    using A = typename acc_of<T>::type;
    Pack v[K][V / N];

    __device__ __forceinline__ A at(int k, int j) const { return (A)v[k][j / N].t[j % N]; }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[k][j / N].t[j % N] = (T)0;
    }

    // Kept as it is: its values are converted where they are used, not once and for all in twice as many registers.
    __device__ __forceinline__ void stay()
    {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V / N; ++i) {
                u4 u = __builtin_bit_cast(u4, v[k][i]);
                asm volatile("" : "+v"(u));
                v[k][i] = __builtin_bit_cast(Pack, u);
            }
    }

    // 0 behind the row's end
    template <bool VEC>
    __device__ __forceinline__ void load(const void *p_, int lane, int group, int cols)
    {
        const T *__restrict__ p = static_cast<const T *>(p_);
        clear();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (VEC) {
                const int c = col_of<true>(k, 0, lane, group);
                if (c < cols)
#pragma unroll
                    for (int i = 0; i < V / N; ++i)
                        v[k][i] = *reinterpret_cast<const Pack *>(p + c + i * N);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int c = col_of<false>(k, j, lane, group);
                    if (c < cols)
                        v[k][j / N].t[j % N] = p[c];
                }
            }
        }
    }
};

template <typename T, int K, bool VEC>
__device__ __forceinline__ void store_row(void *p_, int lane, int group, int cols, const typename acc_of<T>::type (&v)[K][V])
{
    T *__restrict__ p = static_cast<T *>(p_);
    using P = Part<T, K>;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (VEC) {
            const int c = col_of<true>(k, 0, lane, group);
            if (c < cols)
#pragma unroll
                for (int i = 0; i < V / P::N; ++i) {
                    typename P::Pack q;
#pragma unroll
                    for (int j = 0; j < P::N; ++j)
                        q.t[j] = (T)v[k][i * P::N + j];
                    *reinterpret_cast<typename P::Pack *>(p + c + i * P::N) = q;
                }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = col_of<false>(k, j, lane, group);
                if (c < cols)
                    p[c] = (T)v[k][j];
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ const T *row_at(const void *p, long long row, long long ld)
{
    return static_cast<const T *>(p) + row * ld;
}

// Sums over a row's group of threads of N values at once; every thread of the block calls it (rows behind the last one with
// zeros).  Each sum of a row has its own buffer, and rows take two sets of them in turn, so one barrier per sum is enough.
template <typename A, int N>
__device__ __forceinline__ void group_sum(A (&v)[N], int group, A *buf)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = wave_sum(v[i]);
    if (group == 64)
        return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i)
            buf[wave * N + i] = v[i];
    __syncthreads();
    // one load: every sixteen lanes take a sum of each of the group's waves, sixteen at most
    const int per = group >> 6, first = wave / per * per, other = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = other < per ? buf[(first + other) * N + i] : (A)0;
        v[i] = sum_of_16(v[i]);
    }
}

constexpr int kWaves = kMaxThreads / 64;

// for all of a thread's columns
#define FUSE_EACH(...)                                                                                                    \
    do {                                                                                                                  \
        _Pragma("unroll") for (int k = 0; k < K; ++k) _Pragma("unroll") for (int j = 0; j < V; ++j) { __VA_ARGS__; }      \
    } while (0)

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) { return 1.0 / sqrt(v); }

// v[k][j] - mean, 0 behind the row's end
template <bool VEC, bool LAYER, typename A>
__device__ __forceinline__ A centred(A v, A mean, int k, int j, int lane, int group, int cols)
{
    return LAYER ? (col_of<VEC>(k, j, lane, group) < cols ? v - mean : (A)0) : v;
}

// Rows are taken by persistent blocks, a group's next row loaded while this one is worked on; weights stay in registers.
template <typename T, int K, bool VEC, bool LAYER>
__global__ void __launch_bounds__(K < 4 ? 512 : kMaxThreads) block_norm_kernel(const FwdArgs a)
{
    using A = typename acc_of<T>::type;
    __shared__ A buf[2][4][kWaves];
    const int group = a.group, per_block = blockDim.x / group, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / group);
    const int lane = threadIdx.x - mine * group;               // (groups are whole waves: rows are the same for all lanes of one)
    const int cols = a.cols;
    const A scale = (A)a.scale, eps = (A)a.eps;
    Part<T, K> post_w, pre_w, post_b, pre_b, gate, x, z;
    if (a.post_w)
        post_w.template load<VEC>(a.post_w, lane, group, cols);
    if (a.pre_w)
        pre_w.template load<VEC>(a.pre_w, lane, group, cols);
    if (LAYER && a.post_b)
        post_b.template load<VEC>(a.post_b, lane, group, cols);
    if (LAYER && a.pre_b)
        pre_b.template load<VEC>(a.pre_b, lane, group, cols);
    if (a.gate.kind == 1)
        gate.template load<VEC>(a.gate.p, lane, group, cols);
    const long long stride = (long long)gridDim.x * per_block;
    auto load = [&](long long row) {
        if (row < a.rows) {
            x.template load<VEC>(row_at<T>(a.x, row, a.x_ld), lane, group, cols);
            if (a.z)
                z.template load<VEC>(row_at<T>(a.z, row, a.z_ld), lane, group, cols);
        } else {
            x.clear();
            z.clear();
        }
    };
    long long row = (long long)blockIdx.x * per_block + mine;
    load(row);
    for (int turn = 0; row - mine < a.rows; row += stride, turn ^= 1) {
        const bool in = row < a.rows;
        A h[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                h[k][j] = x.at(k, j);
        if (a.z) {
            A u[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    u[k][j] = z.at(k, j);
            if (a.gate.kind == 3 && in)
                gate.template load<VEC>(row_at<T>(a.gate.p, row, a.gate.ld), lane, group, cols);
            A each = scale;
            if (a.gate.kind == 2 && in)
                each *= (A)*row_at<T>(a.gate.p, row, a.gate.ld);
            load(row + stride);
            if (a.post_w) {
                A mean = (A)0, s[1] = {(A)0};
                if (LAYER) {
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            s[0] += u[k][j];
                    group_sum<A, 1>(s, group, buf[turn][0]);
                    mean = s[0] / (A)cols;
                    s[0] = (A)0;
                }
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        u[k][j] = centred<VEC, LAYER>(u[k][j], mean, k, j, lane, group, cols);
                        s[0] += u[k][j] * u[k][j];
                    }
                group_sum<A, 1>(s, group, buf[turn][1]);
                const A r = inv_sqrt(s[0] / (A)cols + eps);
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        u[k][j] = u[k][j] * r * post_w.at(k, j);
                        if (LAYER && a.post_b)
                            u[k][j] += post_b.at(k, j);
                    }
            }
            if (a.gate.kind == 1 || a.gate.kind == 3)
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        u[k][j] *= gate.at(k, j);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    h[k][j] += each * u[k][j];
            if (a.h && in)
                store_row<T, K, VEC>(static_cast<T *>(a.h) + row * a.h_ld, lane, group, cols, h);
        } else {
            load(row + stride);
        }
        if (a.y) {
            // the norm is that of h before its rounding: it is in registers, and y is rounded once
            A mean = (A)0, s[1] = {(A)0};
            if (LAYER) {
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        s[0] += col_of<VEC>(k, j, lane, group) < cols ? h[k][j] : (A)0;
                group_sum<A, 1>(s, group, buf[turn][2]);
                mean = s[0] / (A)cols;
                s[0] = (A)0;
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[k][j] = col_of<VEC>(k, j, lane, group) < cols ? h[k][j] - mean : (A)0;
                    s[0] += h[k][j] * h[k][j];
                }
            group_sum<A, 1>(s, group, buf[turn][3]);
            const A r = inv_sqrt(s[0] / (A)cols + eps);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[k][j] = h[k][j] * r * pre_w.at(k, j);
                    if (LAYER && a.pre_b)
                        h[k][j] += pre_b.at(k, j);
                }
            if (in)
                store_row<T, K, VEC>(static_cast<T *>(a.y) + row * a.y_ld, lane, group, cols, h);
        }
    }
}

// One block's rows of a column sum: the groups of a block are added in order, then the block's partial row is written.
template <typename A, int K, bool VEC>
__device__ __forceinline__ void leave_sum(const A (&v)[K][V], int lane, int mine, int group, int cols, A *out, A *add)
{
    const int per_block = blockDim.x / group;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = col_of<VEC>(k, j, lane, group);
            A s = v[k][j];
            if (per_block > 1) {
                add[threadIdx.x] = s;
                __syncthreads();
                if (mine == 0)
                    for (int g = 1; g < per_block; ++g)
                        s += add[g * group + lane];
                __syncthreads();
            }
            if (mine == 0 && c < cols)
                out[c] = s;
        }
}

// Three sums per row at most: means (layer norms only); squares of h and z and what dy needs of h; what du needs of z.  The row after
// this one is loaded meanwhile.
template <typename T, int K, bool VEC, bool LAYER>
__global__ void __launch_bounds__(K < 4 ? 512 : kMaxThreads, sizeof(T) == 2 && VEC && K == 1 ? 4 : 1) block_norm_grad_kernel(const BwdArgs a)
{
    using A = typename acc_of<T>::type;
    __shared__ A buf[2][3][kWaves * 4];
    __shared__ A add[kMaxThreads];
    const int group = a.group, per_block = blockDim.x / group, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / group);
    const int lane = threadIdx.x - mine * group;               // (groups are whole waves: rows are the same for all lanes of one)
    const int cols = a.cols;
    const A scale = (A)a.scale, eps = (A)a.eps, inv = (A)1 / (A)cols;
    A sum_pre[K][V] = {}, sum_post[K][V] = {}, sum_gate[K][V] = {};
    A sum_pre_b[LAYER ? K : 1][V] = {}, sum_post_b[LAYER ? K : 1][V] = {};
    Part<T, K> post_w, post_b, pre_w, gate, ph, pdy, pdh, pz;
    if (a.post_w)
        post_w.template load<VEC>(a.post_w, lane, group, cols);
    if (LAYER && a.post_b)
        post_b.template load<VEC>(a.post_b, lane, group, cols);
    if (a.pre_w)
        pre_w.template load<VEC>(a.pre_w, lane, group, cols);
    if (a.gate.kind == 1)
        gate.template load<VEC>(a.gate.p, lane, group, cols);
    const long long stride = (long long)gridDim.x * per_block;
    auto load = [&](long long row) {
        const bool in = row < a.rows;
        if (in && a.dy) {
            ph.template load<VEC>(row_at<T>(a.h, row, a.h_ld), lane, group, cols);
            pdy.template load<VEC>(row_at<T>(a.dy, row, a.dy_ld), lane, group, cols);
        } else {
            ph.clear();
            pdy.clear();
        }
        if (in && a.dh)
            pdh.template load<VEC>(row_at<T>(a.dh, row, a.dh_ld), lane, group, cols);
        else
            pdh.clear();
        if (in && a.z)
            pz.template load<VEC>(row_at<T>(a.z, row, a.z_ld), lane, group, cols);
        else
            pz.clear();
    };
    long long row = (long long)blockIdx.x * per_block + mine;
    load(row);
    for (int turn = 0; row - mine < a.rows; row += stride, turn ^= 1) {
        const bool in = row < a.rows;
        if (sizeof(T) == 2) {
            post_w.stay();
            pre_w.stay();
            if (LAYER)
                post_b.stay();
            gate.stay();
        }
        A n[K][V], d[K][V], z[K][V];       // h, then normalised; dy o w, then dx, then the gradient of u; z
        if (a.gate.kind == 3 && in)
            gate.template load<VEC>(row_at<T>(a.gate.p, row, a.gate.ld), lane, group, cols);
        A each = (A)1;
        if (a.gate.kind == 2 && in)
            each = (A)*row_at<T>(a.gate.p, row, a.gate.ld);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                n[k][j] = ph.at(k, j);
                z[k][j] = pz.at(k, j);
                d[k][j] = pdy.at(k, j);
            }
        const Part<T, K> dh = pdh;
        if (K == 1)
            load(row + stride);            // (the registers of longer rows do not hold two of them)
        if (LAYER) {
            A s[2] = {(A)0, (A)0};
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s[0] += n[k][j];
                    s[1] += z[k][j];
                }
            group_sum<A, 2>(s, group, buf[turn][0]);
            const A mh = s[0] / (A)cols, mz = a.post_w ? s[1] / (A)cols : (A)0;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    n[k][j] = centred<VEC, true>(n[k][j], mh, k, j, lane, group, cols);
                    z[k][j] = centred<VEC, true>(z[k][j], mz, k, j, lane, group, cols);
                }
        }
        A s[4] = {(A)0, (A)0, (A)0, (A)0}; // squares of h, squares of z, sum of dy o w o h, sum of dy o w
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[0] += n[k][j] * n[k][j];
                s[1] += z[k][j] * z[k][j];
            }
        if (a.dy) {
            FUSE_EACH(s[2] += d[k][j] * pre_w.at(k, j) * n[k][j]);
            if (LAYER)
                FUSE_EACH(s[3] += d[k][j] * pre_w.at(k, j));
        }
        group_sum<A, 4>(s, group, buf[turn][1]);
        // (a row behind the last one adds 0 to the column sums, eps = 0 included)
        const A rh = in ? inv_sqrt(s[0] / (A)cols + eps) : (A)0, rz = in ? inv_sqrt(s[1] / (A)cols + eps) : (A)0;
        const A with_h = s[2] * rh * inv, with_1 = LAYER ? s[3] * inv : (A)0;
        if (a.dy) {
            FUSE_EACH(n[k][j] *= rh);
            FUSE_EACH(sum_pre[k][j] += d[k][j] * n[k][j]);
            if (LAYER)
                FUSE_EACH(sum_pre_b[LAYER ? k : 0][j] += d[k][j]);
            FUSE_EACH(d[k][j] = rh * (d[k][j] * pre_w.at(k, j) - n[k][j] * with_h - with_1));
        }
        FUSE_EACH(d[k][j] += dh.at(k, j));
        if (in && a.dx)
            store_row<T, K, VEC>(static_cast<T *>(a.dx) + row * a.dx_ld, lane, group, cols, d);
        if (a.z) {
            // d: gradient of u o gate, then of u
            A sz[3] = {(A)0, (A)0, (A)0};  // sum of du o w o z, sum of du o w, sum of the gate's gradient
            const A zs = a.post_w ? rz : (A)1, ds = in ? scale : (A)0;
            FUSE_EACH(d[k][j] = col_of<VEC>(k, j, lane, group) < cols ? d[k][j] * ds : (A)0);
            FUSE_EACH(z[k][j] *= zs);
            A t[K][V];
            if (a.gate.kind != 0) {        // (branches are around the loops, not in them: the same for the whole call)
                FUSE_EACH(t[k][j] = z[k][j]);
                if (a.post_w)
                    FUSE_EACH(t[k][j] *= post_w.at(k, j));
                if (LAYER && a.post_b)
                    FUSE_EACH(t[k][j] += post_b.at(k, j));
                FUSE_EACH(t[k][j] *= d[k][j]);
                if (!in)
                    FUSE_EACH(t[k][j] = (A)0);
                if (a.gate.kind == 1)
                    FUSE_EACH(sum_gate[k][j] += t[k][j]);
                if (a.gate.kind == 2) {
                    FUSE_EACH(sz[2] += t[k][j]);
                    FUSE_EACH(d[k][j] *= each);
                } else if (in) {
                    FUSE_EACH(d[k][j] *= gate.at(k, j));
                }
            }
            if (a.post_w) {
                FUSE_EACH(sum_post[k][j] += d[k][j] * z[k][j]);
                if (LAYER)
                    FUSE_EACH(sum_post_b[LAYER ? k : 0][j] += d[k][j]);
                FUSE_EACH(d[k][j] *= post_w.at(k, j));
                FUSE_EACH(sz[0] += d[k][j] * z[k][j]);
                if (LAYER)
                    FUSE_EACH(sz[1] += d[k][j]);
            }
            if (a.gate.kind == 3 && in && a.dgate)
                store_row<T, K, VEC>(static_cast<T *>(a.dgate) + row * a.dgate_ld, lane, group, cols, t);
            if (a.post_w || a.gate.kind == 2)
                group_sum<A, 3>(sz, group, buf[turn][2]);
            if (a.gate.kind == 2 && a.dgate && in && lane == 0)
                static_cast<T *>(a.dgate)[row * a.dgate_ld] = (T)sz[2];
            if (a.post_w) {
                const A with_z = sz[0] * inv, with_one = LAYER ? sz[1] * inv : (A)0;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        d[k][j] = rz * (d[k][j] - z[k][j] * with_z - with_one);
            }
            if (in && a.dz)
                store_row<T, K, VEC>(static_cast<T *>(a.dz) + row * a.dz_ld, lane, group, cols, d);
        }
        if (K > 1)
            load(row + stride);
    }
    A *out = static_cast<A *>(a.partial) + (long long)blockIdx.x * cols;
    const long long step = (long long)gridDim.x * cols;
    if (a.want_dpre_w)
        leave_sum<A, K, VEC>(sum_pre, lane, mine, group, cols, out, add);
    if (a.want_dpost_w)
        leave_sum<A, K, VEC>(sum_post, lane, mine, group, cols, out + step, add);
    if (a.gate.kind == 1 && a.dgate)
        leave_sum<A, K, VEC>(sum_gate, lane, mine, group, cols, out + 2 * step, add);
    if (LAYER) {
        if (a.want_dpre_b)
            leave_sum<A, LAYER ? K : 1, VEC>(sum_pre_b, lane, mine, group, cols, out + 3 * step, add);
        if (a.want_dpost_b)
            leave_sum<A, LAYER ? K : 1, VEC>(sum_post_b, lane, mine, group, cols, out + 4 * step, add);
    }
}

// Column sums over the blocks' partial rows, in order: 64 columns of one sum per block, 16 slices of the partial rows.
template <typename T>
__global__ void __launch_bounds__(1024) block_norm_sums_kernel(const SumArgs a)
{
    using A = typename acc_of<T>::type;
    __shared__ A part[16][64];
    if (!a.out[blockIdx.y])
        return;
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    const A *p = static_cast<const A *>(a.partial) + (long long)blockIdx.y * a.blocks * a.cols;
    const int per = (a.blocks + 15) / 16, end = min(a.blocks, (slice + 1) * per);
    A s = (A)0;
    if (c < a.cols)
#pragma unroll 8
        for (int b = slice * per; b < end; ++b)
            s += p[(long long)b * a.cols + c];
    part[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && c < a.cols) {
#pragma unroll
        for (int i = 1; i < 16; ++i)
            s += part[i][threadIdx.x & 63];
        static_cast<T *>(a.out[blockIdx.y])[c] = (T)s;
    }
}

// Steps of eight columns per thread, and threads per row: whole waves, as few as that takes.  Blocks of 512 threads leave a thread 256
// registers, which hold a gradient call's sums and two rows of one step each; the longest rows take 1024.
int steps_for(int64_t cols) { return cols <= 512 * V ? 1 : cols <= 1024 * V ? 2 : 4; }

int group_for(int64_t cols)
{
    const int64_t per = 64 * V * steps_for(cols);
    return (int)((cols + per - 1) / per) * 64;
}

// Threads per block: as many groups as 512 hold, at least one.
int threads_for(int64_t cols)
{
    const int g = group_for(cols);
    return g >= 512 ? g : 512 / g * g;
}

int grad_blocks(const fuse_block *b)
{
    const int64_t per = threads_for(b->cols) / group_for(b->cols), want = (b->rows + per - 1) / per;
    return (int)(want < 1 ? 1 : want > kGradBlocks ? kGradBlocks : want);
}

template <typename T, int K, bool VEC>
void launch_fwd_kvl(const FwdArgs &a, bool layer, unsigned blocks, unsigned threads, hipStream_t s)
{
    if (layer)
        block_norm_kernel<T, K, VEC, true><<<blocks, threads, 0, s>>>(a);
    else
        block_norm_kernel<T, K, VEC, false><<<blocks, threads, 0, s>>>(a);
}

template <typename T, int K, bool VEC>
void launch_bwd_kvl(const BwdArgs &a, bool layer, unsigned blocks, unsigned threads, hipStream_t s)
{
    if (layer)
        block_norm_grad_kernel<T, K, VEC, true><<<blocks, threads, 0, s>>>(a);
    else
        block_norm_grad_kernel<T, K, VEC, false><<<blocks, threads, 0, s>>>(a);
}

#define FUSE_BY_STEPS(call, k, vec, ...)                                                                                   \
    do {                                                                                                                  \
        if (vec) {                                                                                                        \
            if (k == 1) call<T, 1, true>(__VA_ARGS__); else if (k == 2) call<T, 2, true>(__VA_ARGS__); else call<T, 4, true>(__VA_ARGS__);     \
        } else {                                                                                                          \
            if (k == 1) call<T, 1, false>(__VA_ARGS__); else if (k == 2) call<T, 2, false>(__VA_ARGS__); else call<T, 4, false>(__VA_ARGS__);  \
        }                                                                                                                 \
    } while (0)

template <typename T>
void launch_fwd(const FwdArgs &a, bool layer, int k, bool vec, unsigned blocks, unsigned threads, hipStream_t s)
{
    FUSE_BY_STEPS(launch_fwd_kvl, k, vec, a, layer, blocks, threads, s);
}

template <typename T>
void launch_bwd(const BwdArgs &a, bool layer, int k, bool vec, unsigned blocks, unsigned threads, hipStream_t s)
{
    FUSE_BY_STEPS(launch_bwd_kvl, k, vec, a, layer, blocks, threads, s);
}

template <typename T>
void launch_sums(const SumArgs &a, hipStream_t s)
{
    block_norm_sums_kernel<T><<<dim3((a.cols + 63) / 64, 5), 1024, 0, s>>>(a);
}

#define FUSE_BY_DTYPE(dtype, call, ...)                                                                                    \
    do {                                                                                                                  \
        switch (dtype) {                                                                                                  \
        case FUSE_F64: call<double>(__VA_ARGS__); break;                                                                  \
        case FUSE_F32: call<float>(__VA_ARGS__); break;                                                                   \
        case FUSE_BF16: call<__bf16>(__VA_ARGS__); break;                                                                 \
        default: call<_Float16>(__VA_ARGS__); break;                                                                      \
        }                                                                                                                 \
    } while (0)

int check_block(const fuse_block *b)
{
    if (!b)
        return report(FUSE_EINVAL, "block is NULL");
    if (!known_dtype(b->dtype))
        return report(FUSE_EINVAL, "dtype is not a fuse_dtype");
    if (b->norm != FUSE_NORM_RMS && b->norm != FUSE_NORM_LAYER)
        return report(FUSE_EINVAL, "norm is not a fuse_norm_kind");
    if (b->rows < 0 || b->cols < 1)
        return report(FUSE_EINVAL, "rows must not be negative and cols must be positive");
    if (b->cols > kMaxCols)
        return report(FUSE_EUNSUPPORTED, "cols " + std::to_string(b->cols) + " > " + std::to_string(kMaxCols));
    if (b->rows > (INT64_C(1) << 40))
        return report(FUSE_EUNSUPPORTED, "rows " + std::to_string(b->rows) + " > 2^40");
    if (!(b->eps >= 0.0))
        return report(FUSE_EINVAL, "eps must not be negative");
    if (!b->z && (b->post_weight || b->gate_kind != FUSE_GATE_NONE))
        return report(FUSE_EINVAL, "a norm after the block and a gate need the block's result z");
    if (b->norm == FUSE_NORM_RMS && (b->post_bias || b->pre_bias))
        return report(FUSE_EINVAL, "a bias needs FUSE_NORM_LAYER");
    if ((b->post_bias && !b->post_weight) || (b->pre_bias && !b->pre_weight))
        return report(FUSE_EINVAL, "a bias needs its norm's weight");
    if (b->gate_kind != FUSE_GATE_NONE && b->gate_kind != FUSE_SIDE_ROWVEC && b->gate_kind != FUSE_SIDE_COLVEC &&
        b->gate_kind != FUSE_SIDE_MATRIX)
        return report(FUSE_EINVAL, "gate_kind is none of FUSE_GATE_NONE, FUSE_SIDE_ROWVEC, FUSE_SIDE_COLVEC, FUSE_SIDE_MATRIX");
    if (b->gate_kind != FUSE_GATE_NONE && !b->gate)
        return report(FUSE_EINVAL, "gate is NULL");
    return FUSE_OK;
}

int check_ld(const fuse_block *b, const void *p, int64_t ld, const char *what)
{
    return p && b->rows > 1 && ld < b->cols ? report(FUSE_ESHAPE, std::string(what) + ": leading dimension < cols") : FUSE_OK;
}

int gate_code(const fuse_block *b)
{
    return b->gate_kind == FUSE_GATE_NONE ? 0 : b->gate_kind == FUSE_SIDE_ROWVEC ? 1 : b->gate_kind == FUSE_SIDE_COLVEC ? 2 : 3;
}

// 16-byte loads: whole rows of vectors, every row of every matrix on 16 bytes.
bool rows_on_16(const fuse_block *b, const void *p, int64_t ld)
{
    return !p || (on_16_bytes(p) && (b->rows <= 1 || (ld * (int64_t)dtype_size(b->dtype)) % 16 == 0));
}

bool block_on_16(const fuse_block *b)
{
    return b->cols % V == 0 && rows_on_16(b, b->z, b->z_ld) && on_16_bytes(b->post_weight) && on_16_bytes(b->post_bias) &&
           on_16_bytes(b->pre_weight) && on_16_bytes(b->pre_bias) &&
           (b->gate_kind == FUSE_GATE_NONE || b->gate_kind == FUSE_SIDE_COLVEC ||
            (b->gate_kind == FUSE_SIDE_ROWVEC ? on_16_bytes(b->gate) : rows_on_16(b, b->gate, b->gate_ld)));
}

int check_gate_ld(const fuse_block *b)
{
    if (b->gate_kind == FUSE_SIDE_MATRIX)
        return check_ld(b, b->gate, b->gate_ld, "gate");
    if (b->gate_kind == FUSE_SIDE_COLVEC && b->rows > 1 && b->gate_ld < 1)
        return report(FUSE_ESHAPE, "gate: stride < 1");
    return FUSE_OK;
}

int norm_impl(const fuse_block *b, const void *x, int64_t x_ld, void *h, int64_t h_ld, void *y, int64_t y_ld, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_block(b);
    if (rc)
        return rc;
    if (b->pre_weight ? !y : y != nullptr)
        return report(FUSE_EINVAL, "y goes with pre_weight: both or neither");
    if (!b->z && h)
        return report(FUSE_EINVAL, "h needs the block's result z: without one it is x");
    if (!h && !y)
        return report(FUSE_EINVAL, "neither h nor y is asked for");
    if (!x && b->rows > 0)
        return report(FUSE_EINVAL, "x is NULL");
    if ((rc = check_ld(b, x, x_ld, "x")) || (rc = check_ld(b, b->z, b->z_ld, "z")) || (rc = check_ld(b, h, h_ld, "h")) ||
        (rc = check_ld(b, y, y_ld, "y")) || (rc = check_gate_ld(b)))
        return rc;
    if (b->rows == 0)
        return FUSE_OK;
    FwdArgs a;
    a.x = x, a.z = b->z, a.post_w = b->post_weight, a.post_b = b->post_bias, a.pre_w = b->pre_weight, a.pre_b = b->pre_bias;
    a.h = h, a.y = y;
    a.x_ld = x_ld, a.z_ld = b->z_ld, a.h_ld = h_ld, a.y_ld = y_ld, a.rows = b->rows;
    a.cols = (int)b->cols, a.group = group_for(b->cols);
    a.gate = {gate_code(b), b->gate, b->gate_ld};
    a.eps = b->eps, a.scale = b->scale;
    const bool vec = block_on_16(b) && rows_on_16(b, x, x_ld) && rows_on_16(b, h, h_ld) && rows_on_16(b, y, y_ld);
    const int threads = threads_for(b->cols), per = threads / a.group;
    const int64_t want = (b->rows + per - 1) / per, most = 256 * (2048 / threads);
    const unsigned blocks = (unsigned)(want > most ? most : want);
    FUSE_BY_DTYPE(b->dtype, launch_fwd, a, b->norm == FUSE_NORM_LAYER, steps_for(b->cols), vec, blocks, threads, (hipStream_t)stream);
    return launched("block_norm_kernel");
}

size_t grad_bytes(const fuse_block *b)
{
    return (size_t)5 * grad_blocks(b) * b->cols * (b->dtype == FUSE_F64 ? 8 : 4);
}

int norm_grad_impl(const fuse_block *b, const void *dh, int64_t dh_ld, const void *dy, int64_t dy_ld, const void *h, int64_t h_ld,
                   const fuse_block_grads *g, void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_block(b);
    if (rc)
        return rc;
    if (!g)
        return report(FUSE_EINVAL, "grads is NULL");
    if (!dh && !dy)
        return report(FUSE_EINVAL, "neither dh nor dy is given");
    if (dy && !b->pre_weight)
        return report(FUSE_EINVAL, "dy needs the norm that made y: pre_weight is NULL");
    if (dy && !h && b->rows > 0)
        return report(FUSE_EINVAL, "h is NULL");
    if (!b->z && g->dz)
        return report(FUSE_EINVAL, "dz needs z");
    if ((g->dgate && b->gate_kind == FUSE_GATE_NONE) || (g->dpost_weight && !b->post_weight) || (g->dpre_weight && !b->pre_weight) ||
        (g->dpost_bias && !b->post_bias) || (g->dpre_bias && !b->pre_bias))
        return report(FUSE_EINVAL, "a gradient is asked for whose input is not given");
    if ((rc = check_ld(b, dh, dh_ld, "dh")) || (rc = check_ld(b, dy, dy_ld, "dy")) || (rc = check_ld(b, h, h_ld, "h")) ||
        (rc = check_ld(b, b->z, b->z_ld, "z")) || (rc = check_ld(b, g->dx, g->dx_ld, "dx")) || (rc = check_ld(b, g->dz, g->dz_ld, "dz")) ||
        (rc = check_gate_ld(b)) ||
        (rc = b->gate_kind == FUSE_SIDE_MATRIX ? check_ld(b, g->dgate, g->dgate_ld, "dgate") : FUSE_OK))
        return rc;
    if (b->gate_kind == FUSE_SIDE_COLVEC && g->dgate && b->rows > 1 && g->dgate_ld < 1)
        return report(FUSE_ESHAPE, "dgate: stride < 1");
    if (!workspace || !on_16_bytes(workspace) || workspace_bytes < grad_bytes(b))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(grad_bytes(b)) + " bytes on 16 are needed");
    BwdArgs a;
    a.dh = dh, a.dy = dy, a.h = h, a.z = b->z, a.post_w = b->post_weight, a.post_b = b->post_bias, a.pre_w = b->pre_weight;
    a.dx = g->dx, a.dz = g->dz, a.dgate = g->dgate, a.partial = workspace;
    a.dh_ld = dh_ld, a.dy_ld = dy_ld, a.h_ld = h_ld, a.z_ld = b->z_ld, a.dx_ld = g->dx_ld, a.dz_ld = g->dz_ld, a.dgate_ld = g->dgate_ld;
    a.rows = b->rows, a.cols = (int)b->cols, a.group = group_for(b->cols);
    a.gate = {gate_code(b), b->gate, b->gate_ld};
    a.eps = b->eps, a.scale = b->scale;
    // (without dy or rows the sums are those of nothing: zeros)
    a.want_dpre_w = g->dpre_weight != nullptr, a.want_dpre_b = g->dpre_bias != nullptr;
    a.want_dpost_w = g->dpost_weight != nullptr, a.want_dpost_b = g->dpost_bias != nullptr;
    const bool vec = block_on_16(b) && rows_on_16(b, dh, dh_ld) && rows_on_16(b, dy, dy_ld) && rows_on_16(b, h, h_ld) &&
                     rows_on_16(b, g->dx, g->dx_ld) && rows_on_16(b, g->dz, g->dz_ld) &&
                     (b->gate_kind != FUSE_SIDE_MATRIX || rows_on_16(b, g->dgate, g->dgate_ld));
    const int blocks = grad_blocks(b);
    FUSE_BY_DTYPE(b->dtype, launch_bwd, a, b->norm == FUSE_NORM_LAYER, steps_for(b->cols), vec, blocks, threads_for(b->cols), (hipStream_t)stream);
    rc = launched("block_norm_grad_kernel");
    SumArgs sa;
    sa.partial = workspace, sa.blocks = blocks, sa.cols = (int)b->cols;
    sa.out[0] = g->dpre_weight, sa.out[1] = g->dpost_weight;
    sa.out[2] = b->gate_kind == FUSE_SIDE_ROWVEC ? g->dgate : nullptr;
    sa.out[3] = g->dpre_bias, sa.out[4] = g->dpost_bias;
    if (rc || (!sa.out[0] && !sa.out[1] && !sa.out[2] && !sa.out[3] && !sa.out[4]))
        return rc;
    FUSE_BY_DTYPE(b->dtype, launch_sums, sa, (hipStream_t)stream);
    rc = launched("block_norm_sums_kernel");
    if (!rc)
        set_last_kernel("block_norm_grad_kernel");
    return rc;
}

}  // namespace

extern "C" {

int fuse_block_norm(const fuse_block *block, const void *x, int64_t x_ld, void *h, int64_t h_ld, void *y, int64_t y_ld, void *stream)
{
    return fuse::guard([&] { return norm_impl(block, x, x_ld, h, h_ld, y, y_ld, stream); });
}

size_t fuse_block_norm_backward_bytes(const fuse_block *block)
{
    if (!block || !known_dtype(block->dtype) || block->rows < 0 || block->cols < 1 || block->cols > kMaxCols)
        return 0;
    return grad_bytes(block);
}

int fuse_block_norm_backward(const fuse_block *block, const void *dh, int64_t dh_ld, const void *dy, int64_t dy_ld, const void *h,
                             int64_t h_ld, const fuse_block_grads *grads, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return norm_grad_impl(block, dh, dh_ld, dy, dy_ld, h, h_ld, grads, workspace, workspace_bytes, stream); });
}

}  // extern "C"
