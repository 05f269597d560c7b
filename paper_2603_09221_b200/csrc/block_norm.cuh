// Norms behind and in front of a block, with its gate, residual scale and residual in one pass over the rows:
//
//     u = x rms_g(x) w_post      rms_g(v) = 1 / sqrt(mean of v^2 over the channels of a group + eps)
//     u = u silu(z)
//     h = r + s u
//     y = h rms(h) w_pre         (one group)
//
// each line where its operand is there.  Backwards, with n = h rms(h), m = x rms_g(x):
//
//     dh += rms(h) (w_pre dy - n mean(n w_pre dy)),  dw_pre = sum n dy;   dr = dh;   ds = sum dh u silu(z)
//     g = s dh:  dz = g u silu'(z);   g = g silu(z):  dw_post = sum g m,  dx = rms_g(x) (w_post g - m mean_g(m w_post g))
//
// Memory bounds both: every operand is read once and every result written once.  A row stays in the registers of the threads that share
// it (a warp, or a block of up to 1024), in vectors of 16 bytes, where its sums are formed in float32.
#pragma once

#include <type_traits>

#include "block_common.cuh"

namespace ttc {
namespace bnorm {

using namespace blk;

constexpr int kRowsOfWarps = 4;                  // rows of a block in which a row is one warp's
constexpr int kAhead = 3;                        // rows whose operands are on their way, gradients

struct NormDev {
    long long rows;
    int d, groups, size;                         // size: channels of a group
    int lanes;                                   // of a group, where that many neighbouring threads share one (a power of two up to 32), else 0
    float eps, per_row, per_group;               // 1 / d, 1 / size
    const void *x, *z, *r, *h_in, *dy, *dh;
    void *h, *y, *dx, *dz, *dr;
    long long ldx, ldz, ldr, ldh, ldy, lddy, lddh, lddx, lddz, lddr;
    const float *w_post, *scale, *w_pre;
    float *dw_post, *dscale, *dw_pre;
    float* parts;                                // [count of row workers][3][d]: shares of dw_post, dscale, dw_pre
    int workers;
    int plain;                                   // h is x
};

extern __shared__ __align__(16) float bnorm_smem[];

// Sums of N values over the threads of a row.  `buffer` [2][32 N]: two take turns, so that one barrier is enough.
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* buffer, int& turn)
{
#pragma unroll
    for (int o = 16; o; o /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (blockDim.x == 32)
        return;
    float* s = buffer + turn * 32 * N;
    turn ^= 1;
    const int warps = blockDim.x / 32, lane = threadIdx.x % 32;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i * 32 + threadIdx.x / 32] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = s[i * 32 + lane % warps];         // (a power of two)
    for (int o = warps / 2; o; o /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

// Sums over the groups of channels: in, the values of a thread's K vectors, one for each element; out, the sum of the element's group.  MIXED: groups that vectors lie across, or of
// more than a warp's vectors, through shared memory, group by group.  Else all elements of a vector have the same sum, and only the first is set: a group is the row, or a few
// neighbouring threads.
template <bool MIXED, int K, int V> __device__ __forceinline__ void group_sums_of(const NormDev& p, float (&v)[K][V], float* area, float* buffer, int& turn)
{
    if constexpr (MIXED) {
        const int warps = blockDim.x / 32;
        float* s = area + threadIdx.y * (p.d + p.groups);
        float* sums = s + p.d;
        __syncthreads();                         // earlier sums have been read
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * blockDim.x + threadIdx.x) * V;
            if (at < p.d)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    s[at + j] = v[k][j];
        }
        __syncthreads();
        for (int g = threadIdx.x / 32; g < p.groups; g += warps) {
            float sum = 0.f;
            for (int j = threadIdx.x % 32; j < p.size; j += 32)
                sum += s[g * p.size + j];
#pragma unroll
            for (int o = 16; o; o /= 2)
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (threadIdx.x % 32 == 0)
                sums[g] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * blockDim.x + threadIdx.x) * V;
            if (at < p.d) {
                int g = at / p.size, left = (g + 1) * p.size - at;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (left == 0) {
                        ++g;
                        left = p.size;
                    }
                    v[k][j] = sums[g];
                    --left;
                }
            }
        }
    } else {
        float all[1] = {0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int j = 1; j < V; ++j)
                v[k][0] += v[k][j];
            all[0] += v[k][0];
        }
        if (p.groups == 1) {
            row_sums<1>(all, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k)
                v[k][0] = all[0];
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int o = 1; o < 32; o *= 2)
                    if (o < p.lanes)
                        v[k][0] += __shfl_xor_sync(0xffffffffu, v[k][0], o);
        }
    }
}

template <typename T, int V> __device__ __forceinline__ void widen(const Vec<T, V>& a, float (&f)[V])
{
    if constexpr (std::is_same<T, bf16>::value && V % 2 == 0) {
        const uint32_t* pairs = reinterpret_cast<const uint32_t*>(&a);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            f[j] = __uint_as_float(pairs[j / 2] << 16);
            f[j + 1] = __uint_as_float(pairs[j / 2] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            f[j] = to_f(a.v[j]);
    }
}
template <typename T, int V> __device__ __forceinline__ void store(T* to, const float (&f)[V])
{
    Vec<T, V> u;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
        uint32_t* pairs = reinterpret_cast<uint32_t*>(&u);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            if constexpr (std::is_same<T, bf16>::value) {
                const __nv_bfloat162 r = __floats2bfloat162_rn(f[j], f[j + 1]);
                pairs[j / 2] = *reinterpret_cast<const uint32_t*>(&r);
            } else {
                const __half2 r = __floats2half2_rn(f[j], f[j + 1]);
                pairs[j / 2] = *reinterpret_cast<const uint32_t*>(&r);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            u.v[j] = from_f<T>(f[j]);
    }
    *reinterpret_cast<Vec<T, V>*>(to) = u;
}
// Parameters of a vector's channels.
template <int V> __device__ __forceinline__ void params(const float* w, int c, bool ok, float (&f)[V])
{
#pragma unroll
    for (int j = 0; j < V; j += V < 4 ? V : 4) {
        const Vec<float, V < 4 ? V : 4> u = load_if(reinterpret_cast<const Vec<float, V < 4 ? V : 4>*>(w + c + j), ok);
#pragma unroll
        for (int i = 0; i < (V < 4 ? V : 4); ++i)
            f[j + i] = u.v[i];
    }
}

template <int V> __device__ __forceinline__ void keep(float* to, const float (&f)[V])
{
#pragma unroll
    for (int j = 0; j < V; j += V < 4 ? V : 4) {
        Vec<float, V < 4 ? V : 4> u;
#pragma unroll
        for (int i = 0; i < (V < 4 ? V : 4); ++i)
            u.v[i] = f[j + i];
        *reinterpret_cast<Vec<float, V < 4 ? V : 4>*>(to + j) = u;
    }
}

// K vectors of V elements to a thread; blockDim.x threads to a row, blockDim.y rows to a block (more than one only where a row is a warp's).
template <typename T, int V, int K, bool MIXED>
__global__ void __launch_bounds__(K < 4 ? 512 : 1024) norm_kernel(const NormDev p)
{
    __shared__ float buffer[2 * 32];
    wait_for_previous();
    const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool here = row < p.rows;
    const int vectors = p.d / V;
    int turn = 0;
    bool ok[K];
    int c[K];
    Vec<T, V> x[K], z[K], r[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = k * blockDim.x + threadIdx.x;
        ok[k] = here && at < vectors;
        c[k] = at < vectors ? at * V : 0;
        const long long lead = here ? row : 0;
        x[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.x) + lead * p.ldx + c[k]), ok[k]);
        z[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.z) + lead * p.ldz + c[k]), ok[k] && p.z);
        r[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.r) + lead * p.ldr + c[k]), ok[k] && p.r);
    }
    float u[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
        widen(x[k], u[k]);
    if (p.w_post) {
        float sum[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[k][j] = u[k][j] * u[k][j];
        group_sums_of<MIXED, K, V>(p, sum, bnorm_smem, buffer, turn);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float w[V];
            params(p.w_post, c[k], true, w);
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[k][j] = MIXED || j == 0 ? rsqrtf(fmaf(sum[k][j], p.per_group, p.eps)) : sum[k][0];
#pragma unroll
            for (int j = 0; j < V; ++j)
                u[k][j] *= sum[k][j] * w[j];
        }
    }
    if (p.z) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float f[V];
            widen(z[k], f);
#pragma unroll
            for (int j = 0; j < V; ++j)
                u[k][j] *= silu(f[j]);
        }
    }
    float square[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (p.scale) {
            float s[V];
            params(p.scale, c[k], true, s);
#pragma unroll
            for (int j = 0; j < V; ++j)
                u[k][j] *= s[j];
        }
        if (p.r) {
            float f[V];
            widen(r[k], f);
#pragma unroll
            for (int j = 0; j < V; ++j)
                u[k][j] += f[j];
        }
        if (p.h && ok[k])
            store<T, V>(static_cast<T*>(p.h) + row * p.ldh + c[k], u[k]);
#pragma unroll
        for (int j = 0; j < V; ++j)
            square[0] = ok[k] ? fmaf(u[k][j], u[k][j], square[0]) : square[0];
    }
    if (!p.w_pre)
        return;
    row_sums<1>(square, buffer, turn);
    const float rms = rsqrtf(fmaf(square[0], p.per_row, p.eps));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float w[V];
        params(p.w_pre, c[k], true, w);
#pragma unroll
        for (int j = 0; j < V; ++j)
            u[k][j] *= rms * w[j];
        if (ok[k])
            store<T, V>(static_cast<T*>(p.y) + row * p.ldy + c[k], u[k]);
    }
}

// Workers (a block, or a warp of one) take every workers-th row and keep their shares of the parameters' gradients in registers.
//
// Where a thread has one vector of each operand of a row, copies of the next rows' vectors into its own places of shared memory are under way (kAhead rows; no other thread looks at
// them), so that memory is at work while the sums of a row are waited for.
template <typename T, int V, int K, bool MIXED>
__global__ void __launch_bounds__(K < 4 ? 512 : 1024) norm_grad_kernel(const NormDev p)
{
    constexpr bool RING = K == 1 && V > 1;
    __shared__ float buffer[2 * 32 * 2];
    wait_for_previous();
    const int worker = blockIdx.x * blockDim.y + threadIdx.y, vectors = p.d / V;
    int turn = 0;
    bool in[K];
    int c[K];
    float s_post[K][V], s_scale[K][V], s_pre[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = k * blockDim.x + threadIdx.x;
        in[k] = at < vectors;
        c[k] = in[k] ? at * V : 0;
#pragma unroll
        for (int j = 0; j < V; ++j)
            s_post[k][j] = s_scale[k][j] = s_pre[k][j] = 0.f;
    }
    const long long rounds = (p.rows + p.workers - 1) / p.workers;               // the same number for all rows of a block: they share barriers
    const int threads = blockDim.x * blockDim.y;
    uint4* ring = reinterpret_cast<uint4*>(bnorm_smem) + threadIdx.y * blockDim.x + threadIdx.x;
    float* area = bnorm_smem + (RING ? kAhead * 5 * threads * 4 : 0);
    int slot = 0;                                // of the ring
    auto ask = [&](long long round) {            // (vectors of nothing where an operand is missing or the row lies behind the last)
        const long long row = round * p.workers + worker;
        const bool ok = in[0] && row < p.rows;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring) + slot * (5 * 16 * threads);
        auto copy = [&](int i, const void* ptr, long long ld, bool there) {
            if (!there && round >= kAhead)       // nothing is there already
                return;
            const bool have = ok && there;
            const T* from = have ? static_cast<const T*>(ptr) + row * ld + c[0] : static_cast<const T*>(p.x);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to + i * (16 * threads)), "l"(from), "r"(have ? 16 : 0) : "memory");
        };
        copy(0, p.x, p.ldx, true);
        copy(1, p.z, p.ldz, p.z);
        copy(2, p.h_in, p.ldh, p.w_pre);
        copy(3, p.dy, p.lddy, p.w_pre);
        copy(4, p.dh, p.lddh, p.dh);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if constexpr (RING) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            ask(i);
            slot = slot + 1 < kAhead ? slot + 1 : 0;
        }
    }
    for (long long round = 0; round < rounds; ++round) {
        const long long row = round * p.workers + worker;
        const bool here = row < p.rows;
        const long long lead = here ? row : 0;
        Vec<T, V> x[K], z[K], h[K], dy[K], dh[K];
        if constexpr (RING) {
            asm volatile("cp.async.wait_group %0;" :: "n"(kAhead - 1) : "memory");
            const uint4* from = ring + slot * 5 * threads;
            x[0] = *reinterpret_cast<const Vec<T, V>*>(from);
            z[0] = *reinterpret_cast<const Vec<T, V>*>(from + threads);
            h[0] = *reinterpret_cast<const Vec<T, V>*>(from + 2 * threads);
            dy[0] = *reinterpret_cast<const Vec<T, V>*>(from + 3 * threads);
            dh[0] = *reinterpret_cast<const Vec<T, V>*>(from + 4 * threads);
            ask(round + kAhead);
            slot = slot + 1 < kAhead ? slot + 1 : 0;
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const bool ok = in[k] && here;
                x[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.x) + lead * p.ldx + c[k]), ok);
                z[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.z) + lead * p.ldz + c[k]), ok && p.z);
                h[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.h_in) + lead * p.ldh + c[k]), ok && p.w_pre);
                dy[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.dy) + lead * p.lddy + c[k]), ok && p.w_pre);
                dh[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.dh) + lead * p.lddh + c[k]), ok && p.dh);
            }
        }
        float g[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k)
            widen(dh[k], g[k]);
        if (p.w_pre) {
            float sums[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V], b[V], w[V];
                widen(h[k], a);
                widen(dy[k], b);
                params(p.w_pre, c[k], true, w);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    sums[0] = fmaf(a[j], a[j], sums[0]);
                    sums[1] = fmaf(a[j], w[j] * b[j], sums[1]);
                }
            }
            row_sums<2>(sums, buffer, turn);
            const float rms = rsqrtf(fmaf(sums[0], p.per_row, p.eps)), mean = sums[1] * p.per_row * rms * rms;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V], b[V], w[V];
                widen(h[k], a);
                widen(dy[k], b);
                params(p.w_pre, c[k], true, w);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s_pre[k][j] = fmaf(a[j] * rms, b[j], s_pre[k][j]);
                    g[k][j] = fmaf(rms, fmaf(w[j], b[j], -a[j] * mean), g[k][j]);
                }
            }
        }
        if (p.dr) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (in[k] && here)
                    store<T, V>(static_cast<T*>(p.dr) + row * p.lddr + c[k], g[k]);
        }
        float inverse[K][V];
        if (p.w_post) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V];
                widen(x[k], a);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    inverse[k][j] = a[j] * a[j];
            }
            group_sums_of<MIXED, K, V>(p, inverse, area, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    inverse[k][j] = MIXED || j == 0 ? rsqrtf(fmaf(inverse[k][j], p.per_group, p.eps)) : inverse[k][0];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float a[V], u[V], gate[V], slope[V], s[V];
            widen(x[k], a);
            if (p.w_post)
                params(p.w_post, c[k], true, u);
            if (p.scale)
                params(p.scale, c[k], true, s);
            if (p.z)
                widen(z[k], slope);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                u[j] = p.w_post ? a[j] * inverse[k][j] * u[j] : a[j];
                gate[j] = 1.f;
                if (p.z) {
                    const float f = slope[j], q = sigmoid(f);
                    gate[j] = f * q;
                    slope[j] = fmaf(q * f, 1.f - q, q);
                }
                if (p.scale) {
                    s_scale[k][j] = fmaf(g[k][j], u[j] * gate[j], s_scale[k][j]);
                    g[k][j] *= s[j];
                }
                if (p.z) {
                    slope[j] *= g[k][j] * u[j];
                    g[k][j] *= gate[j];
                }
            }
            if (p.dz && in[k] && here)
                store<T, V>(static_cast<T*>(p.dz) + row * p.lddz + c[k], slope);
        }
        if (p.w_post) {
            float sum[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V], w[V];
                widen(x[k], a);
                params(p.w_post, c[k], true, w);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s_post[k][j] = fmaf(g[k][j], a[j] * inverse[k][j], s_post[k][j]);
                    g[k][j] *= w[j];
                    sum[k][j] = a[j] * g[k][j];
                }
            }
            group_sums_of<MIXED, K, V>(p, sum, area, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V];
                widen(x[k], a);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float mean = sum[k][MIXED ? j : 0] * p.per_group * inverse[k][j] * inverse[k][j];
                    g[k][j] = inverse[k][j] * fmaf(-a[j], mean, g[k][j]);
                }
            }
        }
        if (p.dx) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (in[k] && here)
                    store<T, V>(static_cast<T*>(p.dx) + row * p.lddx + c[k], g[k]);
        }
    }
    if constexpr (RING)
        asm volatile("cp.async.wait_all;" ::: "memory");
    if (p.parts) {
        float* to = p.parts + (long long)worker * 3 * p.d;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (in[k]) {
                if (p.dw_post)
                    keep(to + c[k], s_post[k]);
                if (p.dscale)
                    keep(to + p.d + c[k], s_scale[k]);
                if (p.dw_pre)
                    keep(to + 2 * p.d + c[k], s_pre[k]);
            }
    }
}

// The workers' shares added up in their order: 32 channels to a block, eight runs of workers side by side.
static __global__ void __launch_bounds__(256) norm_sum_kernel(const NormDev p)
{
    wait_for_previous();
    __shared__ float s[8][32];
    const int lane = threadIdx.x % 32, run = threadIdx.x / 32, which = blockIdx.y, c = blockIdx.x * 32 + lane;
    float* to = which == 0 ? p.dw_post : which == 1 ? p.dscale : p.dw_pre;
    if (!to)
        return;
    float sum = 0.f;
    if (c < p.d) {
        const float* from = p.parts + (long long)which * p.d + c;
        const int lo = (int)((long long)p.workers * run / 8), hi = (int)((long long)p.workers * (run + 1) / 8);
#pragma unroll 8
        for (int w = lo; w < hi; ++w)
            sum += from[(long long)w * 3 * p.d];
    }
    s[run][lane] = sum;
    __syncthreads();
    if (run == 0 && c < p.d) {
        for (int i = 1; i < 8; ++i)
            sum += s[i][lane];
        to[c] = sum;
    }
}

} // namespace bnorm
} // namespace ttc
