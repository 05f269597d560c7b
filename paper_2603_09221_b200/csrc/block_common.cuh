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

// V elements that are loaded and stored together, by 16 bytes where they are more: the alignment that the host sides ask for
template <typename T, int V> struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Vec { T v[V]; };

// First thing in kernels that are launched with launch_early (block_host.h): their blocks are set up while the kernel in front of
// them in the stream ends, and go on once all of it is done and visible; the same is allowed to the kernel behind.
__device__ __forceinline__ void wait_for_previous()
{
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// A load under a predicate, zero without it.  Written out so that no branch is left around it: where two paths join
// behind a load, its result is waited for.
template <typename P> __device__ __forceinline__ P load_if(const P* from, bool ok)
{
    P r;
    if constexpr (sizeof(P) == 16) {
        uint4 v;
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                     "@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}\n"
                     : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(from), "r"((int)ok));
        r = *reinterpret_cast<P*>(&v);
    } else if constexpr (sizeof(P) == 8) {
        uint2 v;
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %3, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\t@p ld.global.v2.b32 {%0, %1}, [%2];\n\t}\n"
                     : "=&r"(v.x), "=&r"(v.y) : "l"(from), "r"((int)ok));
        r = *reinterpret_cast<P*>(&v);
    } else if constexpr (sizeof(P) == 4) {
        uint32_t v;
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.b32 %0, 0;\n\t@p ld.global.b32 %0, [%1];\n\t}\n" : "=&r"(v) : "l"(from), "r"((int)ok));
        r = *reinterpret_cast<P*>(&v);
    } else {
        static_assert(sizeof(P) == 2, "");
        unsigned short v;
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.b16 %0, 0;\n\t@p ld.global.b16 %0, [%1];\n\t}\n" : "=&h"(v) : "l"(from), "r"((int)ok));
        r = *reinterpret_cast<P*>(&v);
    }
    return r;
}

// Stores to shared memory that loads around them may pass: for areas that are only read behind a barrier.  To the compiler an
// ordinary store may touch what the next load reads, and a loop with one in each step waits for its loads step by step.
__device__ __forceinline__ void put_aside(float* to, float a)
{
    asm volatile("st.shared.f32 [%0], %1;" :: "r"((uint32_t)__cvta_generic_to_shared(to)), "f"(a));
}
__device__ __forceinline__ void put_aside(float2* to, float a, float b)
{
    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" :: "r"((uint32_t)__cvta_generic_to_shared(to)), "f"(a), "f"(b));
}
__device__ __forceinline__ void put_aside(float4* to, float a, float b, float c, float d)
{
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"((uint32_t)__cvta_generic_to_shared(to)), "f"(a), "f"(b), "f"(c), "f"(d));
}

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
//
// Exponentials and reciprocals are the special-function unit's (2 u to 4 u, u = 2^-24); the rest is multiply-adds.  The
// arguments -z log2(e) are rounded, which moves exp(-z) by another |z| u.

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Exponents of decays, exp(D A) = 2^(D A log2(e) + kExBias): between -0.2 and 0, where states last, the unit's results fall short by
// 0.5e-8 to 2.2e-8 in the mean, which adds up over the tokens that a state remembers; with the constant the mean error is at most
// 1.2e-8 down to -1 (4.9e-8 below, where a state is forgotten within a few tokens), and 2^kExBias is still 1.
constexpr float kExBias = 2.5e-8f;
__device__ __forceinline__ float rcp(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float sigmoid(float z) { return rcp(1.f + ex2(-z * kLog2e)); }
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }
__device__ __forceinline__ float silu_slope(float z)
{
    const float p = sigmoid(z);
    return fmaf(p * z, 1.f - p, p);
}
// log(1 + exp(z)) = max(z, 0) + log1p(exp(-|z|)), log1p(e) = e P(e) on [0, 1]: P of degree 9, fitted for the relative
// error (4.0e-8 with its coefficients in 32 bits; 1.6e-7 as evaluated)
__device__ constexpr float kLog1p[10] = {1.f, -0.4999990165233612f, 0.3332996368408203f, -0.24954132735729218f, 0.19675931334495544f,
                                         -0.15305569767951965f, 0.10603617131710052f, -0.056959159672260284f, 0.019851263612508774f, -0.0032439809292554855f};
__device__ __forceinline__ float softplus(float z)
{
    const float e = ex2(fabsf(z) * -kLog2e);
    float p = kLog1p[9];
#pragma unroll
    for (int i = 8; i >= 0; --i)
        p = fmaf(p, e, kLog1p[i]);
    return fmaf(p, e, fmaxf(z, 0.f));
}
// Phi(z) and exp(-z^2 / 2): Phi(-|z|) = 1/2 erfcx(|z| / sqrt 2) exp(-z^2 / 2), erfcx as t Q(t), t = 1 / (1 + 0.4 |z| / sqrt 2),
// Q of degree 8, fitted for the relative error (1.7e-7; 4.5e-7 as evaluated): exact in relative terms in the tail too.
__device__ __forceinline__ float normal_cdf(float z, float& bell)
{
    const float a = fabsf(z), t = rcp(fmaf(0.2828427255153656f, a, 1.f));
    bell = ex2(z * z * (-0.5f * kLog2e));
    float q = 0.02512984722852707f;
    q = fmaf(q, t, -0.09144636988639832f);
    q = fmaf(q, t, 0.08453645557165146f);
    q = fmaf(q, t, -0.0027991975657641888f);
    q = fmaf(q, t, 0.07071392983198166f);
    q = fmaf(q, t, 0.08427134901285172f);
    q = fmaf(q, t, 0.1039213165640831f);
    q = fmaf(q, t, 0.11283479630947113f);
    q = fmaf(q, t, 0.11283793300390244f);
    const float tail = q * t * bell;
    return z < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float gelu(float z)
{
    float bell;
    return z * normal_cdf(z, bell);
}

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

// sigmoid, silu and softplus of both: the same operations
__device__ __forceinline__ f2 sigmoid2(f2 z)
{
    float a, b;
    unpack2(mul2(z, pack2(-kLog2e, -kLog2e)), a, b);
    unpack2(add2(pack2(ex2(a), ex2(b)), pack2(1.f, 1.f)), a, b);
    return pack2(rcp(a), rcp(b));
}
__device__ __forceinline__ f2 silu2(f2 z) { return mul2(z, sigmoid2(z)); }
__device__ __forceinline__ f2 softplus2(f2 z)
{
    float a, b;
    unpack2(z, a, b);
    const f2 e = pack2(ex2(fabsf(a) * -kLog2e), ex2(fabsf(b) * -kLog2e));
    f2 p = pack2(kLog1p[9], kLog1p[9]);
#pragma unroll
    for (int i = 8; i >= 0; --i)
        p = fma2(p, e, pack2(kLog1p[i], kLog1p[i]));
    return fma2(p, e, pack2(fmaxf(a, 0.f), fmaxf(b, 0.f)));
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
