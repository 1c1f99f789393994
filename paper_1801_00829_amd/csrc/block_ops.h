// What the statically compiled operators of a transformer block share: element types, errors, wave sums.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>
#include <new>
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
    } catch (const std::bad_alloc &) {
        return report(FUSE_ENOMEM, "out of host memory");
    } catch (const std::exception &ex) {
        return report(FUSE_ERUNTIME, std::string("internal error: ") + ex.what());
    }
}

template <typename A>
__device__ __forceinline__ A wave_sum(A v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o, 64);
    return v;
}

}  // namespace fuse
