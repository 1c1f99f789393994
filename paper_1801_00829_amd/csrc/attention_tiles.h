// Matrix-unit pieces of the attention kernels: operands of the 32 x 32 x 16 product, tiles of rows in LDS.
//
// One product D += A B of a wave: A is 32 x 16, B is 16 x 32.  Lane l (half h = l / 32) holds row l % 32 of A and column l % 32 of
// B, eight neighbours k = 8 h .. 8 h + 7 of each, and of D column l % 32, rows 8 (i / 4) + 4 h + i % 4 for i = 0 .. 15.
//
// All products are taken so that what a wave keeps (its 32 queries, or keys) are columns: S = A B with A from a tile in LDS
// leaves every lane 16 scores of ONE column, so statistics of a column are sums over registers and one exchange between the
// halves, and the scores, rounded, are the B operand of the next product as they lie: element e of half h stands for row
// 4 h + e (e < 4) or 8 + 4 h + e - 4 of sixteen, and A is read in that order.  Its A is the transposed tile, eight rows of one
// column, which the transposing LDS load gives four at a time.
#pragma once
#include "attention.h"

namespace fuse {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> __device__ __forceinline__ f32x16 product(s16x8 a, s16x8 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 product<__bf16>(s16x8 a, s16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 product<_Float16>(s16x8 a, s16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// For the scheduler: N products with an LDS load each, DEPTH loads ahead of the first product.
template <int N, int DEPTH>
__device__ __forceinline__ void ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, DEPTH, 0);
#pragma unroll
    for (int i = 0; i < N - DEPTH; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, DEPTH, 0);
}

// Eight values, rounded, as a B operand.
template <typename T> __device__ __forceinline__ s16x8 rounded(const float *v)
{
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = (T)v[i];
    return __builtin_bit_cast(s16x8, x);
}

// The larger, or the sum, of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float both_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A tile of rows in LDS.  DP: dim rounded up to 64, 96 or 128 (0 behind dim).  Rows of 8 or 16 chunks of 16 bytes; chunk c of row r
// lies in place c ^ turn(r), so that neither the loads of one chunk of 16 neighbouring rows (the A operand of S) nor those of four
// neighbouring chunks of four rows (the transposing load) meet in a bank.
template <int DP>
struct Tile {
    static constexpr int kChunks = DP == 64 ? 8 : 16;      // per row in LDS
    static constexpr int kUsed = DP / 8;
    static constexpr int kRowBytes = kChunks * 16;
    static constexpr int kSteps = DP / 16;                 // products over dim
    static constexpr int kCols = DP / 32;                  // 32 dims each

    static __device__ __forceinline__ int turn(int r)
    {
        return kChunks == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    }

    // Byte offsets of this lane's operands within a tile: rows l % 32 of the plain load, and of the transposing load (dims
    // 32 dt .. of sixteen rows in the order above, first and second four).
    static __device__ __forceinline__ int row_at(int lane, int step)
    {
        const int r = lane & 31, c = step * 2 + (lane >> 5);
        return r * kRowBytes + ((c ^ turn(r)) << 4);
    }
    static __device__ __forceinline__ int col_at(int lane, int dt, int second)
    {
        const int i = lane & 15, r = second * 8 + (lane >> 5) * 4 + (i >> 2);
        const int c = dt * 4 + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
        return r * kRowBytes + ((c ^ turn(r)) << 4) + (i & 1) * 8;
    }
};

__device__ __forceinline__ s16x8 read_row(const char *lds, int at)
{
    return *reinterpret_cast<const s16x8 *>(lds + at);
}

__device__ __forceinline__ s16x8 read_col(const char *lds, int first, int second)
{
    using P = __attribute__((address_space(3))) s16x4 *;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + first));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + second));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Brings ROWS rows of a matrix to LDS by THREADS threads, straight from memory: a wave's load writes 64 chunks one behind the other, so
// each lane asks for the chunk that belongs in its place.  Nothing waits here; the barrier that ends a step waits for the loads.
// Rows from `end` on hold the last row instead: they are masked.  Chunks behind dim are left as they are (clear_tiles).
template <typename T, int DP, int ROWS, int THREADS = 256>
struct Fill {
    using L = Tile<DP>;
    static constexpr int kPerPass = THREADS / L::kChunks, kPasses = ROWS / kPerPass;
    static_assert(kPerPass % 16 == 0 && ROWS % kPerPass == 0, "all rows of a lane have one turn");

    int row, chunk, wave;
    bool in;

    __device__ __forceinline__ explicit Fill(int dim)
    {
        row = threadIdx.x / L::kChunks;
        chunk = (threadIdx.x % L::kChunks) ^ L::turn(row);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        in = chunk * 8 < dim;
    }

    __device__ __forceinline__ void pass(char *lds, int i, const T *from) const
    {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                         (__attribute__((address_space(3))) void *)(lds + i * kPerPass * L::kRowBytes + wave * 1024), 16, 0, 0);
    }

    // `at(r)`: where row r of the matrix is; `first`: the tile's first row, `end` > first
    template <typename F>
    __device__ __forceinline__ void load(char *lds, int first, int end, F at) const
    {
        if (in)
#pragma unroll
            for (int i = 0; i < kPasses; ++i)
                pass(lds, i, at(min(first + row + i * kPerPass, end - 1)) + chunk * 8);
    }

    // A whole tile whose rows lie so that those of one pass are the same distance from the next one's: `tile` its first row, the
    // same for all lanes, `lane` this lane's first element from there (lane_of), `step` the distance.  The addresses are then scalars
    // with one offset per lane, and cost the vector unit nothing.
    __device__ __forceinline__ void load_whole(char *lds, const T *tile, unsigned lane, long long step) const
    {
        if (in)
#pragma unroll
            for (int i = 0; i < kPasses; ++i)
                pass(lds, i, reinterpret_cast<const T *>(reinterpret_cast<const char *>(tile + i * step) + lane));
    }
    __device__ __forceinline__ unsigned lane_of(long long row_at) const { return (unsigned)((row_at + chunk * 8) * (long long)sizeof(T)); }

    __device__ __forceinline__ void load(char *lds, const T *base, long long ld, int first, int end) const
    {
        load(lds, first, end, [=](int r) { return base + r * ld; });
    }
};

// Whether any of `rows` rows of a tile in LDS holds a value that is not finite (0 times it is no number), for a whole wave.  Places that a
// row leaves free (dims of 65 to 96) hold what an earlier block left there and are not looked at: results would depend on it.
template <typename T, int DP>
__device__ __forceinline__ bool holds_no_number(const char *tile, int rows)
{
    float s = 0.0f;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
#pragma clang loop unroll(disable)
    for (int at = lane * 16; at < rows * Tile<DP>::kRowBytes; at += 1024) {
        using L = Tile<DP>;
        typedef T t2 __attribute__((ext_vector_type(2)));
        if (L::kUsed < L::kChunks && (((at >> 4) % L::kChunks) ^ L::turn(at / L::kRowBytes)) >= L::kUsed)
            continue;
        const uint4 v = *reinterpret_cast<const uint4 *>(tile + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const t2 x = __builtin_bit_cast(t2, i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
            s = fmaf((float)x[0], 0.0f, fmaf((float)x[1], 0.0f, s));
        }
    }
    return __any(s != 0.0f);
}

// o += (transposed tile) x weights as the products make it, but pair by pair and without the masked ones.  A masked pair's weight is 0,
// which the matrix units multiply all the same: no number where the tile's value is not finite.  The second run of a block, whose
// first one ended with such results, looks for such values in the steps with a mask and comes here if there are any.
//   weights: the B operands of `rows` rows, [rows / 16][lane], `stride` of them apart; rows low .. high count for this lane's column;
//   d0: the first of the ND times 32 dims.
template <typename T, int DP, int ND>
__device__ __forceinline__ void add_seen(f32x16 (&o)[ND], const char *tile, const s16x8 *weights, int stride, int rows, int low, int high, int d0)
{
    using L = Tile<DP>;
#pragma clang loop unroll(disable)
    for (int r = 0; r < rows; ++r) {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));     // (places are worked out here, where they are needed, and not kept in registers meanwhile)
        const int h = lane >> 5;
        const s16x8 *w8 = weights + (r >> 4) * stride + (lane & 31) + ((r >> 2) & 1) * 32;
        const T w = reinterpret_cast<const T *>(w8)[(r & 3) + ((r >> 3) & 1) * 4];
        if (r < low || r >= high)
            continue;
#pragma unroll
        for (int d = 0; d < ND; ++d)
            if (d0 + d < L::kCols)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = (d0 + d) * 4 + i;        // the chunk of dims 8 c .., of which this half has four
                    const T *v = reinterpret_cast<const T *>(tile + r * L::kRowBytes + ((c ^ L::turn(r)) << 4) + h * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[d][i * 4 + e] = fmaf((float)w, (float)v[e], o[d][i * 4 + e]);
                    __builtin_amdgcn_sched_barrier(0);     // (one after the other: no registers for more, which the products need)
                }
    }
}

// Whether any of the block's four waves says so; `lds`: 16 bytes that nothing is kept in.  Begins and ends as all waves do.
__device__ __forceinline__ bool any_wave(bool v, char *lds)
{
    unsigned *said = reinterpret_cast<unsigned *>(lds);
    const bool mine = __any(v);
    if ((threadIdx.x & 63) == 0)
        said[threadIdx.x >> 6] = mine;
    __syncthreads();
    const uint4 all = *reinterpret_cast<const uint4 *>(lds);
    __syncthreads();
    return (all.x | all.y | all.z | all.w) != 0;
}

// The least of all 256 threads' values, in a scalar register; `lds` as above.
__device__ __forceinline__ int least_of_block(int v, char *lds)
{
    int *said = reinterpret_cast<int *>(lds);
#pragma unroll
    for (int i = 32; i > 0; i >>= 1)
        v = min(v, __shfl_xor(v, i, 64));
    if ((threadIdx.x & 63) == 0)
        said[threadIdx.x >> 6] = v;
    __syncthreads();
    const int4 all = *reinterpret_cast<const int4 *>(lds);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(min(min(all.x, all.y), min(all.z, all.w)));
}

// What this wave has written to LDS may be read by its other lanes.
__device__ __forceinline__ void wave_sees()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Zeros in all places of a kernel's tiles, where some stand for dims behind dim; ends with a barrier.
__device__ __forceinline__ void clear_tiles(char *lds, int bytes)
{
    for (int i = threadIdx.x * 16; i < bytes; i += blockDim.x * 16)
        *reinterpret_cast<uint4 *>(lds + i) = make_uint4(0, 0, 0, 0);
    __syncthreads();
}

// A row of 16-bit values as the B operands of the products over dim: row_of the lane's column, 0 behind dim or without a row.
template <typename T, int DP>
__device__ __forceinline__ void operands(s16x8 (&b)[DP / 16], const T *row, bool in, int dim)
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        b[s] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
        if (in && (s * 2 + h) * 8 < dim)
            b[s] = *reinterpret_cast<const s16x8 *>(row + (s * 2 + h) * 8);
    }
}

// 0 where all of them are finite, no number otherwise
template <int DT>
__device__ __forceinline__ float not_finite(const f32x16 (&o)[DT])
{
    float w = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            w += o[d][i] - o[d][i];
    return w;
}

// A wave's 32 columns of 32 DT dims, rounded, to rows of a matrix.
template <typename T, int DT>
__device__ __forceinline__ void write_columns(const f32x16 (&o)[DT], float f, T *row, int h, int dim)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d * 32 + i * 8 + h * 4 < dim)
                *reinterpret_cast<t4 *>(row + d * 32 + i * 8 + h * 4) =
                    t4{(T)(o[d][i * 4] * f), (T)(o[d][i * 4 + 1] * f), (T)(o[d][i * 4 + 2] * f), (T)(o[d][i * 4 + 3] * f)};
}

}  // namespace fuse
