// The norm of all gradients and their clipping (fuse_grad_norm, fuse_grad_clip): many tensors of mixed types in one launch.
//
//   norm = sqrt(sum over the tensors, sum over their cells, g^2),   out = g * min(1, max_norm / (norm + eps))
//
// Bound by memory: a read for the norm, a read and a write for the clipping.  The list of tensors is a kernel argument (no
// copy to the device, nothing that a captured graph would have to keep), cut into chunks of kChunk cells that the blocks
// take in turn.  Squares and sums are in fp64, whose result it is; every block leaves one partial sum, and whoever needs the
// norm adds the partials in the same order, so that the result does not depend on the order in which blocks finish.
//
// 54 tensors, 700 M cells in bf16 and fp32 (1.4 GB): 271 us for the norm (5.2 TB/s), 480 to 520 us for the clipping (5.4 to 5.8 TB/s).
// Taking the second pass from the end, where the last level's cache may hold what was read last, changes nothing (806 and 802 us).
#include <algorithm>
#include <vector>

#include "block_ops.h"

namespace {

using namespace fuse;

constexpr int kTensors = 128;              // tensors per launch: the list stays within 4 KB of kernel arguments
constexpr int kChunk = 8192;               // cells: 16 or more bytes in flight for every thread, four times over
constexpr int kBlocks = 2048;              // per launch; eight blocks of 256 threads fill a compute unit

struct Table {
    const void *p[kTensors];
    void *out[kTensors];                   // NULL: in place
    long long cells[kTensors];
    int chunk0[kTensors];                  // first chunk of every tensor
    unsigned char dtype[kTensors];
    int n, chunks;
};

__device__ __forceinline__ int tensor_of(const Table &t, int chunk)
{
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.chunk0[mid] <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Sum over the block's 256 threads, the same value in every thread; `part` is read before the next barrier only.
__device__ __forceinline__ double block_sum(double v, double *part)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename T>
__device__ __forceinline__ double squares(const T *__restrict__ p, long long cells)
{
    constexpr int N = 16 / sizeof(T);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
        struct alignas(16) Pack { T t[N]; };
        const Pack *q = reinterpret_cast<const Pack *>(p);
        const int packs = (int)(cells / N);
        int i = threadIdx.x;
        for (; i + 768 < packs; i += 1024) {
            Pack v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = q[i + u * 256];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const double d = (double)(typename acc_of<T>::type)v[u].t[j];
                    s[u] = fma(d, d, s[u]);
                }
        }
        for (; i < packs; i += 256) {
            const Pack v = q[i];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const double d = (double)(typename acc_of<T>::type)v.t[j];
                s[j & 3] = fma(d, d, s[j & 3]);
            }
        }
        const int rest = packs * N + threadIdx.x;
        if (rest < cells) {
            const double d = (double)(typename acc_of<T>::type)p[rest];
            s[0] = fma(d, d, s[0]);
        }
    } else {
        for (int i = threadIdx.x; i < cells; i += 256) {
            const double d = (double)(typename acc_of<T>::type)p[i];
            s[0] = fma(d, d, s[0]);
        }
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ void __launch_bounds__(256) grad_squares_kernel(const Table t, double *__restrict__ partial)
{
    __shared__ double part[4];
    double s = 0.0;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int i = tensor_of(t, c);
        const long long first = (long long)(c - t.chunk0[i]) * kChunk, left = t.cells[i] - first;
        const long long cells = left < kChunk ? left : kChunk;
        switch (t.dtype[i]) {
        case FUSE_F64: s += squares(static_cast<const double *>(t.p[i]) + first, cells); break;
        case FUSE_F32: s += squares(static_cast<const float *>(t.p[i]) + first, cells); break;
        case FUSE_BF16: s += squares(static_cast<const __bf16 *>(t.p[i]) + first, cells); break;
        default: s += squares(static_cast<const _Float16 *>(t.p[i]) + first, cells); break;
        }
    }
    s = block_sum(s, part);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = s;
}

// The norm from the partial sums, by one block of 256 threads.
__device__ __forceinline__ double norm_from(const double *__restrict__ partial, int count, double *part)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += 256)
        s += partial[i];
    return sqrt(block_sum(s, part));
}

__global__ void __launch_bounds__(256) grad_norm_kernel(const double *__restrict__ partial, int count, double *__restrict__ norm)
{
    __shared__ double part[4];
    const double s = norm_from(partial, count, part);
    if (threadIdx.x == 0)
        norm[0] = s;
}

template <typename T>
__device__ __forceinline__ void scaled(const T *p, T *out, long long cells, typename acc_of<T>::type f)
{
    using A = typename acc_of<T>::type;
    constexpr int N = 16 / sizeof(T);
    if (((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0) {
        struct alignas(16) Pack { T t[N]; };
        const Pack *q = reinterpret_cast<const Pack *>(p);
        Pack *o = reinterpret_cast<Pack *>(out);
        const int packs = (int)(cells / N);
        int i = threadIdx.x;
        for (; i + 768 < packs; i += 1024) {
            Pack v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = q[i + u * 256];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    v[u].t[j] = (T)((A)v[u].t[j] * f);
                o[i + u * 256] = v[u];
            }
        }
        for (; i < packs; i += 256) {
            Pack v = q[i];
#pragma unroll
            for (int j = 0; j < N; ++j)
                v.t[j] = (T)((A)v.t[j] * f);
            o[i] = v;
        }
        const int rest = packs * N + threadIdx.x;
        if (rest < cells)
            out[rest] = (T)((A)p[rest] * f);
    } else {
        for (int i = threadIdx.x; i < cells; i += 256)
            out[i] = (T)((A)p[i] * f);
    }
}

// count >= 0: the norm is taken from that many partial sums (every block adds them: a few KB from L2, instead of a launch
// of its own), and block 0 of the first launch leaves it in norm_out.  count < 0: the norm is norm_in[0].
__global__ void __launch_bounds__(256) grad_scale_kernel(const Table t, const double *__restrict__ partial, int count,
                                                         const double *__restrict__ norm_in, double *__restrict__ norm_out,
                                                         double max_norm, double eps)
{
    __shared__ double part[4];
    const double norm = count < 0 ? norm_in[0] : norm_from(partial, count, part);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0)
        norm_out[0] = norm;
    const double q = max_norm / (norm + eps), f = q < 1.0 || q != q ? q : 1.0;       // (a norm that is no number makes none of all)
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int i = tensor_of(t, c);
        if (f == 1.0 && t.out[i] == t.p[i])
            continue;                      // in place and short enough: nothing changes
        const long long first = (long long)(c - t.chunk0[i]) * kChunk, left = t.cells[i] - first;
        const long long cells = left < kChunk ? left : kChunk;
        switch (t.dtype[i]) {
        case FUSE_F64: scaled(static_cast<const double *>(t.p[i]) + first, static_cast<double *>(t.out[i]) + first, cells, f); break;
        case FUSE_F32: scaled(static_cast<const float *>(t.p[i]) + first, static_cast<float *>(t.out[i]) + first, cells, (float)f); break;
        case FUSE_BF16: scaled(static_cast<const __bf16 *>(t.p[i]) + first, static_cast<__bf16 *>(t.out[i]) + first, cells, (float)f); break;
        default: scaled(static_cast<const _Float16 *>(t.p[i]) + first, static_cast<_Float16 *>(t.out[i]) + first, cells, (float)f); break;
        }
    }
}

int check_list(const fuse_tensor *tensors, int64_t n)
{
    if (n < 0 || (n > 0 && !tensors))
        return report(FUSE_EINVAL, "tensors is NULL or their number negative");
    for (int64_t i = 0; i < n; ++i) {
        const std::string which = "tensor " + std::to_string(i) + ": ";
        if (!known_dtype(tensors[i].dtype))
            return report(FUSE_EINVAL, which + "dtype is not a fuse_dtype");
        if (tensors[i].count < 0 || (tensors[i].count > 0 && !tensors[i].data))
            return report(FUSE_EINVAL, which + "data is NULL or count negative");
        if (reinterpret_cast<uintptr_t>(tensors[i].data) % dtype_size(tensors[i].dtype) ||
            reinterpret_cast<uintptr_t>(tensors[i].out) % dtype_size(tensors[i].dtype))
            return report(FUSE_EINVAL, which + "data or out is not aligned to its type");
        if (tensors[i].count > (INT64_C(1) << 42))
            return report(FUSE_EUNSUPPORTED, which + "count > 2^42");
    }
    return FUSE_OK;
}

// Blocks write in no order: an output must not meet another output, nor the data of a tensor other than its own.
int check_overlap(const fuse_tensor *tensors, int64_t n)
{
    struct Range { uintptr_t from, to; int64_t tensor; bool out; };
    std::vector<Range> r;
    r.reserve((size_t)n * 2);
    for (int64_t i = 0; i < n; ++i) {
        const fuse_tensor &x = tensors[i];
        const size_t bytes = (size_t)x.count * dtype_size(x.dtype);
        if (!bytes)
            continue;
        const uintptr_t p = reinterpret_cast<uintptr_t>(x.data), o = x.out ? reinterpret_cast<uintptr_t>(x.out) : p;
        r.push_back({o, o + bytes, i, true});
        if (o != p)
            r.push_back({p, p + bytes, i, false});
    }
    std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.from < b.from; });
    uintptr_t out_end = 0, any_end = 0;
    int64_t out_of = 0, any_of = 0;
    for (const Range &x : r) {
        if (x.from < out_end || (x.out && x.from < any_end))
            return report(FUSE_EINVAL, "tensor " + std::to_string(x.tensor) + " overlaps tensor " +
                          std::to_string(x.from < out_end ? out_of : any_of) + " where one of them is written");
        if (x.to > any_end)
            any_end = x.to, any_of = x.tensor;
        if (x.out)
            out_end = x.to, out_of = x.tensor;
    }
    return FUSE_OK;
}

// The norm is read, or written, while tensors are: it must not lie in one that is written, nor be written into one that is read.
int check_norm(const fuse_tensor *tensors, int64_t n, const double *norm, bool written)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(norm);
    if (p % sizeof(double))
        return report(FUSE_EINVAL, "the norm is not aligned to its type");
    for (int64_t i = 0; i < n; ++i) {
        const size_t bytes = (size_t)tensors[i].count * dtype_size(tensors[i].dtype);
        const uintptr_t d = reinterpret_cast<uintptr_t>(tensors[i].data), o = tensors[i].out ? reinterpret_cast<uintptr_t>(tensors[i].out) : d;
        if ((p < o + bytes && o < p + sizeof(double)) || (written && p < d + bytes && d < p + sizeof(double)))
            return report(FUSE_EINVAL, "the norm overlaps tensor " + std::to_string(i));
    }
    return FUSE_OK;
}

// The next launch's tensors, from tensor `at` and its cell `from` on; false: none are left.  A launch takes at most 2^30
// chunks, so a longer tensor is continued by the next one.
bool next_table(const fuse_tensor *tensors, int64_t n, int64_t &at, int64_t &from, Table &t)
{
    constexpr int64_t kMost = INT64_C(1) << 30;
    t.n = 0;
    int64_t chunks = 0;
    while (at < n && t.n < kTensors && chunks < kMost) {
        const fuse_tensor &x = tensors[at];
        int64_t left = x.count - from;
        if (left > (kMost - chunks) * kChunk)
            left = (kMost - chunks) * kChunk;
        if (left > 0) {
            const size_t skip = (size_t)from * dtype_size(x.dtype);
            t.p[t.n] = static_cast<const char *>(x.data) + skip;
            t.out[t.n] = static_cast<char *>(x.out ? x.out : const_cast<void *>(x.data)) + skip;
            t.cells[t.n] = left;
            t.chunk0[t.n] = (int)chunks;
            t.dtype[t.n] = (unsigned char)x.dtype;
            ++t.n;
            chunks += (left + kChunk - 1) / kChunk;
        }
        from += left;
        if (from >= x.count) {
            ++at;
            from = 0;
        }
    }
    t.chunks = (int)chunks;
    return t.n > 0;
}

unsigned blocks_of(const Table &t) { return (unsigned)(t.chunks < kBlocks ? t.chunks : kBlocks); }

// Launches and partial sums of a list.
void extent(const fuse_tensor *tensors, int64_t n, int64_t &partials)
{
    Table t;
    int64_t at = 0, from = 0;
    partials = 0;
    while (next_table(tensors, n, at, from, t))
        partials += blocks_of(t);
}

int squares_of(const fuse_tensor *tensors, int64_t n, double *partial, hipStream_t s, int &count)
{
    Table t;
    int64_t at = 0, from = 0;
    count = 0;
    while (next_table(tensors, n, at, from, t)) {
        grad_squares_kernel<<<blocks_of(t), 256, 0, s>>>(t, partial + count);
        if (const int rc = launched("grad_squares_kernel"))
            return rc;
        count += (int)blocks_of(t);
    }
    return FUSE_OK;
}

int check_workspace(const fuse_tensor *tensors, int64_t n, const void *workspace, size_t bytes)
{
    int64_t partials;
    extent(tensors, n, partials);
    if (partials > (1 << 30))
        return report(FUSE_EUNSUPPORTED, "too many tensors");
    if (partials && (!workspace || !on_16_bytes(workspace) || bytes < (size_t)partials * sizeof(double)))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(partials * sizeof(double)) + " bytes on 16 are needed");
    return FUSE_OK;
}

int grad_norm_impl(const fuse_tensor *tensors, int64_t n, double *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_list(tensors, n);
    if (rc)
        return rc;
    if (!norm)
        return report(FUSE_EINVAL, "norm is NULL");
    if ((rc = check_workspace(tensors, n, workspace, workspace_bytes)))
        return rc;
    int count = 0;
    if ((rc = squares_of(tensors, n, static_cast<double *>(workspace), (hipStream_t)stream, count)))
        return rc;
    grad_norm_kernel<<<1, 256, 0, (hipStream_t)stream>>>(static_cast<double *>(workspace), count, norm);
    return launched("grad_norm_kernel");
}

int grad_clip_impl(const fuse_tensor *tensors, int64_t n, double max_norm, double eps, const double *norm_in, double *norm_out,
                   void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_list(tensors, n);
    if (rc)
        return rc;
    if ((rc = check_overlap(tensors, n)))
        return rc;
    if (!(max_norm >= 0.0) || !(eps >= 0.0))
        return report(FUSE_EINVAL, "max_norm and eps must not be negative");
    if (norm_in ? norm_out != nullptr : !norm_out)
        return report(FUSE_EINVAL, "one of norm_in and norm_out is needed");
    hipStream_t s = (hipStream_t)stream;
    int count = -1;
    if (!norm_in && (rc = check_workspace(tensors, n, workspace, workspace_bytes)))
        return rc;
    if ((rc = check_norm(tensors, n, norm_in ? norm_in : norm_out, !norm_in)))
        return rc;
    if (!norm_in) {
        if ((rc = squares_of(tensors, n, static_cast<double *>(workspace), s, count)))
            return rc;
        if (count == 0) {                  // no cells at all: a norm of 0 and nothing to clip
            grad_norm_kernel<<<1, 256, 0, s>>>(static_cast<double *>(workspace), 0, norm_out);
            return launched("grad_norm_kernel");
        }
        if (count > kBlocks) {             // several launches: the partial sums are added once, not by every block
            grad_norm_kernel<<<1, 256, 0, s>>>(static_cast<double *>(workspace), count, norm_out);
            if ((rc = launched("grad_norm_kernel")))
                return rc;
            norm_in = norm_out;
            norm_out = nullptr;
            count = -1;
        }
    }
    Table t;
    int64_t at = 0, from = 0;
    while (next_table(tensors, n, at, from, t)) {
        grad_scale_kernel<<<blocks_of(t), 256, 0, s>>>(t, static_cast<const double *>(workspace), count, norm_in, norm_out, max_norm, eps);
        if ((rc = launched("grad_scale_kernel")))
            return rc;
        norm_out = nullptr;
    }
    return FUSE_OK;
}

}  // namespace

extern "C" {

size_t fuse_grad_norm_bytes(const fuse_tensor *tensors, int64_t n)
{
    int64_t partials = 0;
    if (n < 0 || (n > 0 && !tensors))
        return 0;
    for (int64_t i = 0; i < n; ++i)
        if (!known_dtype(tensors[i].dtype) || tensors[i].count < 0 || tensors[i].count > (INT64_C(1) << 42))
            return 0;
    extent(tensors, n, partials);
    return (size_t)partials * sizeof(double);
}

int fuse_grad_norm(const fuse_tensor *tensors, int64_t n, double *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return grad_norm_impl(tensors, n, norm, workspace, workspace_bytes, stream); });
}

int fuse_grad_clip(const fuse_tensor *tensors, int64_t n, double max_norm, double eps, const double *norm_in, double *norm_out,
                   void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] {
        return grad_clip_impl(tensors, n, max_norm, eps, norm_in, norm_out, workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
