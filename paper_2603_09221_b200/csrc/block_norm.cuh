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

#include "block_common.cuh"

namespace ttc {
namespace bnorm {

using namespace blk;

constexpr int kRowsOfWarps = 4;                  // rows of a block in which a row is one warp's

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

extern __shared__ float bnorm_smem[];

// Sums of N values over the threads of a row.  `buffer` [2][32 N]: two take turns, so that one barrier is enough.
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* buffer, int& turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o; o /= 2)
            v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (blockDim.x == 32)
        return;
    float* s = buffer + turn * 32 * N;
    turn ^= 1;
    const int warps = blockDim.x / 32;
    if (threadIdx.x % 32 == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[threadIdx.x / 32 * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.f;
        for (int w = 0; w < warps; ++w)
            v[i] += s[w * N + i];
    }
}

// Sums over the groups of channels, of N values for each of a thread's K vectors.  Where a group is a few neighbouring threads, among them; else
// through shared memory, group by group.
template <int N, int K, int V> __device__ __forceinline__ void group_sums_of(const NormDev& p, float (&v)[K][N], float* buffer, int& turn)
{
    if (p.groups == 1) {
        float all[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            all[i] = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
                all[i] += v[k][i];
        }
        row_sums<N>(all, buffer, turn);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[k][i] = all[i];
        return;
    }
    if (p.lanes) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int o = 1; o < 32; o *= 2)
                    if (o < p.lanes)
                        v[k][i] += __shfl_xor_sync(0xffffffffu, v[k][i], o);
        return;
    }
    // one area for each row of the block: [N][vectors], then [N][groups]
    const int vectors = p.d / V, each = vectors + p.groups, warps = blockDim.x / 32, per_group = p.size / V;
    float* s = bnorm_smem + threadIdx.y * N * each;
    float* sums = s + N * vectors;
    __syncthreads();                             // earlier sums have been read
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = k * blockDim.x + threadIdx.x;
        if (at < vectors)
#pragma unroll
            for (int i = 0; i < N; ++i)
                s[i * vectors + at] = v[k][i];
    }
    __syncthreads();
    for (int g = threadIdx.x / 32; g < p.groups; g += warps)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float sum = 0.f;
            for (int j = threadIdx.x % 32; j < per_group; j += 32)
                sum += s[i * vectors + g * per_group + j];
#pragma unroll
            for (int o = 16; o; o /= 2)
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (threadIdx.x % 32 == 0)
                sums[i * p.groups + g] = sum;
        }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = k * blockDim.x + threadIdx.x;
        if (at < vectors)
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[k][i] = sums[i * p.groups + at / per_group];
    }
}

template <typename T, int V> __device__ __forceinline__ void widen(const Vec<T, V>& a, float (&f)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j)
        f[j] = to_f(a.v[j]);
}
template <typename T, int V> __device__ __forceinline__ void store(T* to, const float (&f)[V])
{
    Vec<T, V> u;
#pragma unroll
    for (int j = 0; j < V; ++j)
        u.v[j] = from_f<T>(f[j]);
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
template <typename T, int V, int K>
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
        float sum[K][1];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            sum[k][0] = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[k][0] = fmaf(u[k][j], u[k][j], sum[k][0]);
        }
        group_sums_of<1, K, V>(p, sum, buffer, turn);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float rms = rsqrtf(fmaf(sum[k][0], p.per_group, p.eps));
            float w[V];
            params(p.w_post, c[k], true, w);
#pragma unroll
            for (int j = 0; j < V; ++j)
                u[k][j] *= rms * w[j];
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
template <typename T, int V, int K>
__global__ void __launch_bounds__(K < 4 ? 512 : 1024) norm_grad_kernel(const NormDev p)
{
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
    for (long long round = 0; round < rounds; ++round) {
        const long long row = round * p.workers + worker;
        const bool here = row < p.rows;
        const long long lead = here ? row : 0;
        Vec<T, V> x[K], z[K], h[K], dy[K], dh[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool ok = in[k] && here;
            x[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.x) + lead * p.ldx + c[k]), ok);
            z[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.z) + lead * p.ldz + c[k]), ok && p.z);
            h[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.h_in) + lead * p.ldh + c[k]), ok && p.w_pre);
            dy[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.dy) + lead * p.lddy + c[k]), ok && p.w_pre);
            dh[k] = load_if(reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.dh) + lead * p.lddh + c[k]), ok && p.dh);
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
        float inverse[K];
        if (p.w_post) {
            float sum[K][1];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V];
                widen(x[k], a);
                sum[k][0] = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    sum[k][0] = fmaf(a[j], a[j], sum[k][0]);
            }
            group_sums_of<1, K, V>(p, sum, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k)
                inverse[k] = rsqrtf(fmaf(sum[k][0], p.per_group, p.eps));
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
                u[j] = p.w_post ? a[j] * inverse[k] * u[j] : a[j];
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
            float sum[K][1];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V], w[V];
                widen(x[k], a);
                params(p.w_post, c[k], true, w);
                sum[k][0] = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s_post[k][j] = fmaf(g[k][j], a[j] * inverse[k], s_post[k][j]);
                    g[k][j] *= w[j];
                    sum[k][0] = fmaf(a[j], g[k][j], sum[k][0]);
                }
            }
            group_sums_of<1, K, V>(p, sum, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float a[V];
                widen(x[k], a);
                const float mean = sum[k][0] * p.per_group * inverse[k] * inverse[k];
#pragma unroll
                for (int j = 0; j < V; ++j)
                    g[k][j] = inverse[k] * fmaf(-a[j], mean, g[k][j]);
            }
        }
        if (p.dx) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (in[k] && here)
                    store<T, V>(static_cast<T*>(p.dx) + row * p.lddx + c[k], g[k]);
        }
    }
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
