// What the statically compiled operators of a transformer block share: element types, errors, wave sums.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "../../include/fuse.h"
#include "runtime.h"

namespace fuse {

// Sums, statistics and element-wise arithmetic of a type: fp64 for fp64, fp32 for the others.
template <typename T> struct acc_of { using type = float; };
template <> struct acc_of<double> { using type = double; };

inline size_t dtype_size(int dtype)
{
    return dtype == FUSE_F64 ? 8 : dtype == FUSE_F32 ? 4 : 2;
}

inline bool known_dtype(int dtype) { return dtype >= FUSE_F64 && dtype <= FUSE_F16; }

inline bool on_16_bytes(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether the launch before this call was accepted.
inline int launched(const char *kernel)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return report(FUSE_ERUNTIME, std::string(kernel) + ": " + hipGetErrorString(e));
    set_last_kernel(kernel);
    return FUSE_OK;
}

// No C++ exception may cross the C boundary.
template <typename F>
int guard(F f)
{
    try {
        return f();
    } catch (...) {
        return report_exception();
    }
}

// The same for calls that return a number of bytes: 0.
template <typename F>
size_t guard_bytes(F f)
{
    size_t n = 0;
    return guard([&] { n = f(); return FUSE_OK; }) == FUSE_OK ? n : 0;
}

// v of another lane of the same sixteen, by the pattern CTRL (a move within the registers: no LDS latency).
template <int CTRL>
__device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double moved(double v)
{
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, true),
                            __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, true));
}

// Sum over each sixteen lanes, in all of them: neighbours, pairs, halves of eight and of sixteen.
template <typename A>
__device__ __forceinline__ A sum_of_16(A v)
{
    v += moved<0xB1>(v);                   // lanes 1 0 3 2
    v += moved<0x4E>(v);                   // lanes 2 3 0 1
    v += moved<0x141>(v);                  // mirrored within eight
    v += moved<0x140>(v);                  // mirrored within sixteen
    return v;
}

// Sum of the two values that a swap of v with itself leaves: v of lane l and of the lane 16, or 32, away.
template <int WIDTH>
__device__ __forceinline__ float swapped_sum(float v)
{
    const unsigned u = __float_as_uint(v);
    const auto r = WIDTH == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int WIDTH>
__device__ __forceinline__ double swapped_sum(double v)
{
    const unsigned lo = (unsigned)__double2loint(v), hi = (unsigned)__double2hiint(v);
    const auto l = WIDTH == 16 ? __builtin_amdgcn_permlane16_swap(lo, lo, false, false) : __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
    const auto h = WIDTH == 16 ? __builtin_amdgcn_permlane16_swap(hi, hi, false, false) : __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}

template <typename A>
__device__ __forceinline__ A wave_sum(A v)
{
    return swapped_sum<32>(swapped_sum<16>(sum_of_16(v)));
}

}  // namespace fuse
