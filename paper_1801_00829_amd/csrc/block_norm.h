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
// Bound by memory: a row is read once and, up to 8192 columns (fp64: 4096, gradients 2048), stays in registers through all its statistics.
// A group of G threads owns a row, 16 bytes of it per thread and step, so a row of up to 4096 columns of a 16 bit type is one step.  Longer
// rows take the form of 32 columns per thread, whose blocks of up to 1024 threads leave 128 registers each: most of a row then goes through
// scratch memory, 630 to 1820 bytes per lane (fp64: 2.1 to 3.9 KB; 100 to 1150 from 2048 or 4096 columns on), and this is what bounds these
// rows.  Statistics of a layer norm are taken in two passes over the registers (mean, then squares of the differences): one pass of sums of
// squares would lose the digits that a large mean has.
//
// 16384 x 4096 bf16, a norm on both sides and a gate per column: forward 102 us (5.3 TB/s), gradient 170 + 5 us (4.6 TB/s); a large copy
// reaches 4.7 to 5.4 TB/s on the same card.  Of as many cells (forward, gradient; TB/s): 8192 columns 4.4, 3.5; 8200 columns 0.7, 0.5;
// 12288, 16384 and 32768 columns 1.0, 0.5 to 0.6; fp32 of 12288 columns 1.1, 1.0; fp64 of 4096, 8192 and 16384 (layer) columns 5.1, 3.6 /
// 3.6, 2.0 / 0.6, 0.4; layer norms in bf16 of 4096 columns 4.5, 2.2, of 8192 columns 4.5, 3.0.  What it took: the next row loaded ahead
// (119 -> 101 us forward), sums by moves within the registers instead of LDS (gradient 246 -> 203), branches around the columns' loops (203
// -> 182), the next row asked for before the first sum (182 -> 167).  Rows that are not on 16 bytes: 5003 x 1111 fp32, layer norms with a
// gate per cell, gradient 51 us (3.5 TB/s); 16380 x 4097 bf16, as above: forward 183 us (2.9 TB/s), gradient 359 us (2.2 TB/s).
#pragma once
#include <algorithm>
#include <atomic>

#include "block_ops.h"

namespace fuse {

// Columns per thread and step: 16 bytes of a row, 32 of fp64.
template <typename T> constexpr int kEach = sizeof(T) == 2 ? 8 : 4;
constexpr int kMaxCols = 32768;            // 1024 threads, 32 columns each
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
template <bool VEC, int V>
__device__ __forceinline__ int col_of(int k, int j, int lane, int group)
{
    return VEC ? (k * group + lane) * V + j : (k * V + j) * group + lane;
}

// A thread's part of a row as it lies in memory: what is loaded ahead of its use stays in the row's own type.
template <typename T, int K>
struct Part {
    struct alignas(16) Pack { T t[16 / sizeof(T)]; };
    static constexpr int V = kEach<T>, N = 16 / sizeof(T);
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
                const int c = col_of<true, V>(k, 0, lane, group);
                if (c < cols)
#pragma unroll
                    for (int i = 0; i < V / N; ++i)
                        v[k][i] = *reinterpret_cast<const Pack *>(p + c + i * N);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int c = col_of<false, V>(k, j, lane, group);
                    if (c < cols)
                        v[k][j / N].t[j % N] = p[c];
                }
            }
        }
    }
};

template <typename T, int K, bool VEC>
__device__ __forceinline__ void store_row(void *p_, int lane, int group, int cols, const typename acc_of<T>::type (&v)[K][kEach<T>])
{
    constexpr int V = kEach<T>;
    T *__restrict__ p = static_cast<T *>(p_);
    using P = Part<T, K>;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (VEC) {
            const int c = col_of<true, V>(k, 0, lane, group);
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
                const int c = col_of<false, V>(k, j, lane, group);
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
template <bool VEC, bool LAYER, int V, typename A>
__device__ __forceinline__ A centred(A v, A mean, int k, int j, int lane, int group, int cols)
{
    return LAYER ? (col_of<VEC, V>(k, j, lane, group) < cols ? v - mean : (A)0) : v;
}

// Rows are taken by persistent blocks, a group's next row loaded while this one is worked on; weights stay in registers.
template <typename T, int K, bool VEC, bool LAYER>
__global__ void __launch_bounds__(K * kEach<T> < 32 ? 512 : kMaxThreads) block_norm_kernel(const FwdArgs a)
{
    using A = typename acc_of<T>::type;
    constexpr int V = kEach<T>;
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
                        u[k][j] = centred<VEC, LAYER, V>(u[k][j], mean, k, j, lane, group, cols);
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
                        s[0] += col_of<VEC, V>(k, j, lane, group) < cols ? h[k][j] : (A)0;
                group_sum<A, 1>(s, group, buf[turn][2]);
                mean = s[0] / (A)cols;
                s[0] = (A)0;
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[k][j] = col_of<VEC, V>(k, j, lane, group) < cols ? h[k][j] - mean : (A)0;
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
template <typename A, int K, int V, bool VEC>
__device__ __forceinline__ void leave_sum(const A (&v)[K][V], int lane, int mine, int group, int cols, A *out, A *add)
{
    const int per_block = blockDim.x / group;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = col_of<VEC, V>(k, j, lane, group);
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

// (Two blocks per compute unit for 16 bit types, which takes 128 registers: so does LAYER, with 72 bytes per lane in scratch memory in bf16
// and 40 in fp16; 16384 x 4096 bf16: 360 us.)
//
// Three sums per row at most: means (layer norms only); squares of h and z and what dy needs of h; what du needs of z.  The row after
// this one is loaded meanwhile.
template <typename T, int K, bool VEC, bool LAYER>
__global__ void __launch_bounds__(K * kEach<T> < 32 ? 512 : kMaxThreads, sizeof(T) == 2 && VEC && K == 1 ? 4 : 1) block_norm_grad_kernel(const BwdArgs a)
{
    using A = typename acc_of<T>::type;
    constexpr int V = kEach<T>;
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
        if (K * V <= 8)
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
                    n[k][j] = centred<VEC, true, V>(n[k][j], mh, k, j, lane, group, cols);
                    z[k][j] = centred<VEC, true, V>(z[k][j], mz, k, j, lane, group, cols);
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
            FUSE_EACH(d[k][j] = col_of<VEC, V>(k, j, lane, group) < cols ? d[k][j] * ds : (A)0);
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
        if (K * V > 8)
            load(row + stride);
    }
    A *out = static_cast<A *>(a.partial) + (long long)blockIdx.x * cols;
    const long long step = (long long)gridDim.x * cols;
    if (a.want_dpre_w)
        leave_sum<A, K, V, VEC>(sum_pre, lane, mine, group, cols, out, add);
    if (a.want_dpost_w)
        leave_sum<A, K, V, VEC>(sum_post, lane, mine, group, cols, out + step, add);
    if (a.gate.kind == 1 && a.dgate)
        leave_sum<A, K, V, VEC>(sum_gate, lane, mine, group, cols, out + 2 * step, add);
    if (LAYER) {
        if (a.want_dpre_b)
            leave_sum<A, LAYER ? K : 1, V, VEC>(sum_pre_b, lane, mine, group, cols, out + 3 * step, add);
        if (a.want_dpost_b)
            leave_sum<A, LAYER ? K : 1, V, VEC>(sum_post_b, lane, mine, group, cols, out + 4 * step, add);
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

// Persistent blocks: as many as the device holds at once (asked for once per kernel and block size), so that all of them run from
// start to end; a few more would run when the others are done.
template <auto KERNEL>
unsigned resident_blocks(unsigned threads)
{
    static std::atomic<int> known[kMaxThreads / 64 + 1];
    std::atomic<int> &n = known[threads / 64];
    if (!n.load(std::memory_order_relaxed)) {
        int per = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per, KERNEL, (int)threads, 0) != hipSuccess || per < 1) {
            (void)hipGetLastError();
            per = 1;
        }
        n.store(per, std::memory_order_relaxed);
    }
    return (unsigned)(n.load(std::memory_order_relaxed) * Runtime::get().num_cus());
}

// A type's kernels by steps per row and alignment (see steps_for); `most` blocks where all of them are resident.
#define FUSE_BY_STEPS(kernel, a, layer, k, vec, most, threads, s)                                                          \
    do {                                                                                                                  \
        if (vec) {                                                                                                        \
            if (layer) FUSE_STEPS(kernel, k, true, true, a, most, threads, s); else FUSE_STEPS(kernel, k, true, false, a, most, threads, s);     \
        } else {                                                                                                          \
            if (layer) FUSE_STEPS(kernel, k, false, true, a, most, threads, s); else FUSE_STEPS(kernel, k, false, false, a, most, threads, s);   \
        }                                                                                                                 \
    } while (0)
#define FUSE_STEPS(kernel, k, vec, layer, a, most, threads, s)                                                             \
    do {                                                                                                                  \
        if (k == 1) FUSE_PERSISTENT((kernel<T, 1, vec, layer>), a, most, threads, s);                                     \
        else if (k == 2) FUSE_PERSISTENT((kernel<T, 2, vec, layer>), a, most, threads, s);                                \
        else if (k == 4) FUSE_PERSISTENT((kernel<T, 4, vec, layer>), a, most, threads, s);                                \
        else FUSE_PERSISTENT((kernel<T, 32 / kEach<T>, vec, layer>), a, most, threads, s);                                \
    } while (0)
#define FUSE_PERSISTENT(kernel, a, most, threads, s)                                                                       \
    kernel<<<std::min(most, resident_blocks<kernel>(threads)), threads, 0, s>>>(a)

template <typename T>
void launch_fwd(const FwdArgs &a, bool layer, int k, bool vec, unsigned most, unsigned threads, hipStream_t s)
{
    FUSE_BY_STEPS(block_norm_kernel, a, layer, k, vec, most, threads, s);
}

// (a gradient call's blocks are those that its workspace has room for)
template <typename T>
void launch_bwd(const BwdArgs &a, bool layer, int k, bool vec, unsigned blocks, unsigned threads, hipStream_t s)
{
#define FUSE_GRAD(k_, vec_, layer_) block_norm_grad_kernel<T, k_, vec_, layer_><<<blocks, threads, 0, s>>>(a)
#define FUSE_GRAD_STEPS(vec_, layer_)                                                                                      \
    do {                                                                                                                  \
        if (k == 1) FUSE_GRAD(1, vec_, layer_);                                                                           \
        else if (k == 2) FUSE_GRAD(2, vec_, layer_);                                                                      \
        else if (k == 4) FUSE_GRAD(4, vec_, layer_);                                                                      \
        else FUSE_GRAD(32 / kEach<T>, vec_, layer_);                                                                      \
    } while (0)
    if (vec) {
        if (layer) FUSE_GRAD_STEPS(true, true); else FUSE_GRAD_STEPS(true, false);
    } else {
        if (layer) FUSE_GRAD_STEPS(false, true); else FUSE_GRAD_STEPS(false, false);
    }
#undef FUSE_GRAD
#undef FUSE_GRAD_STEPS
}

template <typename T>
void launch_sums(const SumArgs &a, hipStream_t s)
{
    block_norm_sums_kernel<T><<<dim3((a.cols + 63) / 64, 5), 1024, 0, s>>>(a);
}

// Each type is compiled by a source of its own (block_norm_<type>.hip), side by side.
#define FUSE_NORM_TYPE(prefix, T)                                                                                          \
    prefix template void launch_fwd<T>(const FwdArgs &, bool, int, bool, unsigned, unsigned, hipStream_t);                \
    prefix template void launch_bwd<T>(const BwdArgs &, bool, int, bool, unsigned, unsigned, hipStream_t);                \
    prefix template void launch_sums<T>(const SumArgs &, hipStream_t);

}  // namespace fuse
