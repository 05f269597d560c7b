// What the host sides of the operators of include/ttc_block.h share: checks of arguments, the device of a call, scratch.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/ttc_block.h"
#include "block_common.cuh"
#include "status.h"

namespace ttc {
namespace blk {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - (1 << 16);    // token and offset arithmetic of a sequence fits 32 bits
constexpr int kMaxGridY = 65535;

// Makes `device` current for the duration of a call.
struct DeviceScope {
    int before = -1;
    bool changed = false;
    int enter(int device)
    {
        TTC_CUDA(cudaGetDevice(&before));
        if (before != device) {
            TTC_CUDA(cudaSetDevice(device));
            changed = true;
        }
        return TTC_OK;
    }
    ~DeviceScope()
    {
        if (changed)
            cudaSetDevice(before);
    }
};

// Multiprocessors of a device (148 where it cannot be asked: sizes of scratch are then those of a B200).
inline int sm_count(int device)
{
    static std::atomic<int> known[64];
    if (device < 0 || device >= 64)
        return 148;
    int n = known[device].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            return 148;
        }
        known[device].store(n, std::memory_order_relaxed);
    }
    return n;
}

inline size_t element_size(int dtype) { return dtype == TTC_F32 ? 4 : 2; }

inline int check_dtype(int dtype, bool f32)
{
    if (dtype == TTC_BF16 || dtype == TTC_F16 || (f32 && dtype == TTC_F32))
        return TTC_OK;
    return fail(TTC_STATUS_INVALID_ARGUMENT, "element type %d not supported", dtype);
}

inline int check_rows(const char* name, const ttc_rows& r, int dtype, bool optional)
{
    if (!r.ptr) {
        if (optional)
            return TTC_OK;
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s is null", name);
    }
    if (reinterpret_cast<uintptr_t>(r.ptr) % element_size(dtype))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s is not aligned to its elements", name);
    if (r.bstride < 0 || r.tstride < 0)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s: negative stride", name);
    return TTC_OK;
}

inline int check_floats(const char* name, const void* p, bool optional, size_t align = 4)
{
    if (!p && !optional)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s is null", name);
    if (reinterpret_cast<uintptr_t>(p) % align)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s is not aligned to its elements", name);
    return TTC_OK;
}

inline int check_sequences(int64_t batch, int64_t tokens, const int32_t* offsets)
{
    if (batch < 0 || tokens < 0)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "batch %lld, tokens %lld", (long long)batch, (long long)tokens);
    if (batch > kMaxRows || tokens > kMaxRows || (!offsets && batch && tokens > kMaxRows / batch))
        return fail(TTC_STATUS_UNSUPPORTED, "more than %lld rows", (long long)kMaxRows);
    return check_floats("seq_offsets", offsets, true);
}

inline Rows dev_rows(const ttc_rows& r, const int32_t* offsets) { return Rows{r.ptr, offsets ? 0 : r.bstride, r.tstride}; }

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }

// Rows of an output and of an input that share elements, or may.  Where the strides are the same, they share one if the distance
// of their first elements is i S + j s + c for differences i, j of sequences and tokens and c of columns: for each i (S the larger
// stride: few come into question) the j that leaves the least c is looked at.  Other strides, or rows that overlap one another
// so often that i is not soon found: ranges that meet.
inline bool rows_overlap(const ttc_rows& a, int64_t wa, const ttc_rows& b, int64_t wb, int64_t batch, int64_t tokens, bool packed, size_t size)
{
    if (!a.ptr || !b.ptr || batch <= 0 || tokens <= 0)
        return false;
    const int64_t nb = packed ? 0 : batch - 1, nt = tokens - 1;
    const char *a0 = static_cast<const char*>(a.ptr), *b0 = static_cast<const char*>(b.ptr);
    const char* a1 = a0 + (nb * a.bstride + nt * a.tstride + wa) * (int64_t)size;
    const char* b1 = b0 + (nb * b.bstride + nt * b.tstride + wb) * (int64_t)size;
    if (a1 <= b0 || b1 <= a0)
        return false;
    if ((nt > 0 && a.tstride != b.tstride) || (nb > 0 && a.bstride != b.bstride))
        return true;
    int64_t S = nt > 0 ? a.tstride : 0, nS = nt, s = nb > 0 ? a.bstride : 0, ns = nb;
    if (S < s) {
        const int64_t t = S, n = nS;
        S = s, nS = ns, s = t, ns = n;
    }
    const int64_t far = (b0 - a0) / (int64_t)size, least = 1 - wb, most = wa - 1;               // c in least .. most
    int64_t i0 = 0, i1 = 0;
    if (S > 0) {
        i0 = -floor_div(most + ns * s - far, S), i1 = floor_div(far - least + ns * s, S);
        i0 = i0 < -nS ? -nS : i0, i1 = i1 > nS ? nS : i1;
    }
    if (i1 - i0 > 64)
        return true;
    for (int64_t i = i0; i <= i1; ++i) {
        const int64_t left = far - i * S;
        int64_t j = s > 0 ? floor_div(left - least, s) : 0;
        j = j > ns ? ns : j;
        const int64_t c = left - j * s;
        if (j >= -ns && c >= least && c <= most)
            return true;
    }
    return false;
}

inline bool ranges_meet(const void* a, size_t bytes_a, const void* b, size_t bytes_b)
{
    const char *a0 = static_cast<const char*>(a), *b0 = static_cast<const char*>(b);
    return a0 && b0 && a0 < b0 + bytes_b && b0 < a0 + bytes_a;
}

// Parts of a workspace, each aligned to 256 bytes.
struct Scratch {
    char* base;
    size_t used = 0;
    explicit Scratch(void* p) : base(static_cast<char*>(p)) {}
    template <typename T> T* take(size_t count)
    {
        T* r = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += (count * sizeof(T) + 255) / 256 * 256;
        return r;
    }
};

inline int check_workspace(const void* ws, int64_t have, size_t need)
{
    if (need == 0)
        return TTC_OK;
    if (!ws || have < (int64_t)need)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "workspace of %lld bytes, %zu are needed", ws ? (long long)have : 0ll, need);
    if (reinterpret_cast<uintptr_t>(ws) % 256)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "workspace is not aligned to 256 bytes");
    return TTC_OK;
}

#define TTC_TRY(expr)            \
    do {                         \
        const int s_ = (expr);   \
        if (s_ != TTC_OK)        \
            return s_;           \
    } while (0)

inline int launched(const char* what)
{
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TTC_OK : fail(TTC_STATUS_CUDA_ERROR, "%s: %s", what, cudaGetErrorString(e));
}

// Launch of a kernel that begins with wait_for_previous: what a launch costs behind another one (about 1 us) overlaps with that
// one's end (a projection of 8 rows, 4.7 us: 6.1 -> 5.0 us a call).  For kernels of few blocks and those with one block on every SM:
// blocks that come while another kernel ends gather on the SMs that it leaves first, which cost the scan of 128 blocks 154 -> 192 us
// and the convolution of 4 x 2048 x 4096 34.8 -> 37.5.
// `cluster`: blocks of a cluster, along y.
template <typename... P, typename... A>
int launch_early(const char* what, void (*kernel)(P...), dim3 grid, int threads, int smem, int cluster, cudaStream_t st, const A&... args)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute with[2];
    with[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    with[0].val.programmaticStreamSerializationAllowed = 1;
    with[1].id = cudaLaunchAttributeClusterDimension;
    with[1].val.clusterDim.x = with[1].val.clusterDim.z = 1;
    with[1].val.clusterDim.y = cluster;
    c.attrs = with;
    c.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, P(args)...);
    return e == cudaSuccess ? launched(what) : fail(TTC_STATUS_CUDA_ERROR, "%s: %s", what, cudaGetErrorString(e));
}

// Calls f with a value of the element type.
template <typename F> int by_type(int dtype, F&& f)
{
    switch (dtype) {
    case TTC_F32: return f(float());
    case TTC_BF16: return f(bf16());
    default: return f(__half());
    }
}

} // namespace blk
} // namespace ttc
