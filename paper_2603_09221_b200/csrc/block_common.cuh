// What the operators of include/ttc_block.h share on the device: element types, token rows, packed pairs of floats.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ttc_block.h"

namespace ttc {
namespace blk {

typedef __nv_bfloat16 bf16;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// V elements that are loaded and stored together
template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

struct Rows {
    void* ptr;
    long long bs, ts;
};

template <typename T> __device__ __forceinline__ T* row_ptr(const Rows& r, long long seq, long long row)
{
    return static_cast<T*>(r.ptr) + seq * r.bs + row * r.ts;
}

// The sequences of a call.  Equal: offsets null, rows of sequence b are addressed as (b, t).  Packed: every row is
// addressed as (0, row); the host has set bstride to 0.
struct Seqs {
    const int* offsets;
    long long batch, tokens;
};

struct Span {
    long long row0;   // row of the sequence's first token
    long long len;
};

__device__ __forceinline__ long long clamp_offset(const Seqs& s, long long b)
{
    long long o = s.offsets[b];
    return o < 0 ? 0 : o > s.tokens ? s.tokens : o;
}

__device__ __forceinline__ Span span_of(const Seqs& s, long long b)
{
    if (!s.offsets)
        return Span{0, s.tokens};
    long long lo = clamp_offset(s, b), hi = clamp_offset(s, b + 1);
    return Span{lo, hi > lo ? hi - lo : 0};
}

// ---- activations ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
__device__ __forceinline__ float silu(float z) { return z / (1.f + expf(-z)); }
__device__ __forceinline__ float silu_slope(float z)
{
    float p = sigmoid(z);
    return p * (1.f + z * (1.f - p));
}
__device__ __forceinline__ float softplus(float z) { return fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))); }

// ---- pairs of floats: one instruction for two lanes of arithmetic ------------------------------------------------------

typedef unsigned long long f2;

__device__ __forceinline__ f2 pack2(float a, float b)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float sum2(f2 v)
{
    float a, b;
    unpack2(v, a, b);
    return a + b;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Sums over the W lanes of a group (lanes that differ in the bits STRIDE, 2 STRIDE, .. of the lane index).  In: NV values
// of every lane.  While a lane holds more than one value, a round sends half of them to the partner and keeps the sums of
// the other half; after that the rest is added up.  Afterwards lane j of the group holds in v[0 .. NV / min(NV, W)) the
// sums of values first_value<NV, W>(j) + i.
template <int NV, int W, int STRIDE> __device__ __forceinline__ void group_sums(float (&v)[NV], int lane)
{
    int have = NV;
#pragma unroll
    for (int bit = 1; bit < W; bit *= 2) {
        const int o = bit * STRIDE;
        if (have > 1) {
            have /= 2;
            const bool upper = lane & o;
#pragma unroll
            for (int i = 0; i < NV / 2; ++i)
                if (i < have) {
                    const float send = upper ? v[i] : v[i + have], keep = upper ? v[i + have] : v[i];
                    v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
}
template <int NV, int W> __host__ __device__ __forceinline__ int first_value(int j)
{
    int first = 0, have = NV;
    for (int bit = 1; bit < W && have > 1; bit *= 2) {
        have /= 2;
        first += j & bit ? have : 0;
    }
    return first;
}

} // namespace blk
} // namespace ttc
