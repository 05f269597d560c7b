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
// it (a warp, or a block of up to 1024), in vectors of 16 bytes, where its sums are formed in float32.  Measured, and at the rate that copies reach: forward, 8192 x 4096 bfloat16 with every
// part 61 us, 51; gradients, 8192 x 2048 of all of them 77, 41 (instructions: 56 % of the issue slots), 4093 x 1000 in groups of 125 channels in float32 41, 13; 8 rows 2.6 us, two rounds
// of loads.
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
};

extern __shared__ __align__(16) float bnorm_smem[];

constexpr int kSlot = 2 * 32;                    // of two values over 32 warps

// Sums of N values (one or two) over the threads of a row.  `buffer` [2][kSlot]: two take turns, so that one barrier is enough.  They lie apart whatever N is: calls
// of one and of two values take turns on the same buffer.
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* buffer, int& turn)
{
    static_assert(32 * N <= kSlot, "");
#pragma unroll
    for (int o = 16; o; o /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (blockDim.x == 32)
        return;
    float* s = buffer + turn * kSlot;
    turn ^= 1;
    const int warps = blockDim.x / 32, lane = threadIdx.x % 32, span = 1 << (32 - __clz(warps - 1));       // (warps: two at least)
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i * 32 + threadIdx.x / 32] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = (lane & (span - 1)) < warps ? s[i * 32 + (lane & (span - 1))] : 0.f;
    for (int o = span / 2; o; o /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

// ---- the vectors of a thread as pairs of floats (one instruction for two lanes of arithmetic; a single element's partner is nothing) ----

template <int V> constexpr int kPairs = (V + 1) / 2;

__device__ __forceinline__ f2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float sum_of(f2 v)
{
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

template <typename T, int V> __device__ __forceinline__ void widen(const Vec<T, V>& a, f2 (&f)[kPairs<V>])
{
    if constexpr (V == 1) {
        f[0] = pack2(to_f(a.v[0]), 0.f);
    } else if constexpr (std::is_same<T, bf16>::value) {
        const uint32_t* pairs = reinterpret_cast<const uint32_t*>(&a);
#pragma unroll
        for (int j = 0; j < V / 2; ++j)
            f[j] = pack2(__uint_as_float(pairs[j] << 16), __uint_as_float(pairs[j] & 0xffff0000u));
    } else {
#pragma unroll
        for (int j = 0; j < V / 2; ++j)
            f[j] = pack2(to_f(a.v[2 * j]), to_f(a.v[2 * j + 1]));
    }
}
template <typename T, int V> __device__ __forceinline__ void store(T* to, const f2 (&f)[kPairs<V>])
{
    Vec<T, V> u;
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) {
        float a, b;
        unpack2(f[j], a, b);
        if constexpr (V == 1) {
            u.v[0] = from_f<T>(a);
        } else if constexpr (std::is_same<T, bf16>::value) {
            const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
            reinterpret_cast<uint32_t*>(&u)[j] = *reinterpret_cast<const uint32_t*>(&r);
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 r = __floats2half2_rn(a, b);
            reinterpret_cast<uint32_t*>(&u)[j] = *reinterpret_cast<const uint32_t*>(&r);
        } else {
            u.v[2 * j] = a;
            u.v[2 * j + 1] = b;
        }
    }
    *reinterpret_cast<Vec<T, V>*>(to) = u;
}
// Parameters of a vector's channels.
template <int V> __device__ __forceinline__ void params(const float* w, int c, f2 (&f)[kPairs<V>])
{
    if constexpr (V == 1) {
        f[0] = pack2(w[c], 0.f);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 u = *reinterpret_cast<const float4*>(w + c + j);
            f[j / 2] = pack2(u.x, u.y);
            f[j / 2 + 1] = pack2(u.z, u.w);
        }
    }
}

// How groups of channels lie: a group is the row or neighbouring threads' vectors, a power of two of them up to 32; vectors lie across groups; vectors lie in one each, of which the
// sums alone go through shared memory (gradients of 13541 x 1216 in two groups 170 -> 145 us).
enum { kNear = 0, kAcross = 1, kWhole = 2 };

// Sums over the groups of channels: in, the values of a thread's K vectors; out, the sum of each element's group.  MIXED: groups that vectors lie across, or of
// more than a warp's vectors, through shared memory, group by group.  Else all elements of a vector have the same sum, and only the first pair is set: a group is the row, or a few
// neighbouring threads.
template <int MIXED, int K, int V> __device__ __forceinline__ void group_sums_of(const NormDev& p, f2 (&v)[K][kPairs<V>], float* area, float* buffer, int& turn)
{
    if constexpr (MIXED) {
        const int warps = blockDim.x / 32;
        float* s = area + threadIdx.y * (p.d + p.groups);
        float* sums = s + p.d;
        constexpr bool whole = MIXED == kWhole;
        const int size = whole ? p.size / V : p.size;
        __syncthreads();                         // earlier sums have been read
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * blockDim.x + threadIdx.x) * V;
            if (whole && at < p.d) {
                f2 sum = v[k][0];
#pragma unroll
                for (int j = 1; j < kPairs<V>; ++j)
                    sum = add2(sum, v[k][j]);
                s[at / V] = sum_of(sum);
            } else if (at < p.d) {
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    float a, b;
                    unpack2(v[k][j / 2], a, b);
                    s[at + j] = a;
                    if (V > 1)
                        s[at + j + (V > 1)] = b;
                }
            }
        }
        __syncthreads();
        for (int g = threadIdx.x / 32; g < p.groups; g += warps) {
            float sum = 0.f;
            for (int j = threadIdx.x % 32; j < size; j += 32)
                sum += s[g * size + j];
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
            if (whole && at < p.d) {
                const f2 sum = both(sums[at / p.size]);
#pragma unroll
                for (int j = 0; j < kPairs<V>; ++j)
                    v[k][j] = sum;
            } else if (at < p.d) {
                int g = at / p.size, left = (g + 1) * p.size - at;
                float e[2];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (left == 0) {
                        ++g;
                        left = p.size;
                    }
                    e[j & 1] = sums[g];
                    --left;
                    if ((j & 1) || V == 1)
                        v[k][j / 2] = pack2(e[0], V == 1 ? e[0] : e[1]);
                }
            }
        }
    } else {
        float one[K], all[1] = {0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            f2 sum = v[k][0];
#pragma unroll
            for (int j = 1; j < kPairs<V>; ++j)
                sum = add2(sum, v[k][j]);
            one[k] = sum_of(sum);
            all[0] += one[k];
        }
        if (p.groups == 1) {
            row_sums<1>(all, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k)
                v[k][0] = both(all[0]);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int o = 1; o < 32; o *= 2)
                    if (o < p.lanes)
                        one[k] += __shfl_xor_sync(0xffffffffu, one[k], o);
                v[k][0] = both(one[k]);
            }
        }
    }
}
// 1 / sqrt(sum / size + eps), from what group_sums_of leaves.
template <int MIXED, int V> __device__ __forceinline__ void inverse_roots(f2 (&v)[kPairs<V>], float per_group, float eps)
{
#pragma unroll
    for (int j = 0; j < (MIXED ? kPairs<V> : 1); ++j) {
        float a, b;
        unpack2(v[j], a, b);
        a = rsqrtf(fmaf(a, per_group, eps));
        v[j] = MIXED ? pack2(a, rsqrtf(fmaf(b, per_group, eps))) : both(a);
    }
#pragma unroll
    for (int j = 1; j < kPairs<V>; ++j)
        v[j] = MIXED ? v[j] : v[0];
}

template <int V> __device__ __forceinline__ void keep(float* to, const f2 (&v)[kPairs<V>])
{
    float f[2 * kPairs<V>];
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j)
        unpack2(v[j], f[2 * j], f[2 * j + 1]);
#pragma unroll
    for (int j = 0; j < V; j += V < 4 ? V : 4) {
        Vec<float, V < 4 ? V : 4> u;
#pragma unroll
        for (int i = 0; i < (V < 4 ? V : 4); ++i)
            u.v[i] = f[j + i];
        *reinterpret_cast<Vec<float, V < 4 ? V : 4>*>(to + j) = u;
    }
}

// K vectors of V elements to a thread; blockDim.x threads to a row, blockDim.y rows to a block (more than one only where a row is a warp's).  Pairs of floats: 68 -> 60 us with every part.
template <typename T, int V, int K, int MIXED>
__global__ void __launch_bounds__(K < 4 || V == 8 ? 512 : 1024) norm_kernel(const NormDev p)
{
    __shared__ float buffer[2 * kSlot];
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
    constexpr int P = kPairs<V>;
    f2 u[K][P];
#pragma unroll
    for (int k = 0; k < K; ++k)
        widen(x[k], u[k]);
    if (p.w_post) {
        f2 sum[K][P];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < P; ++j)
                sum[k][j] = mul2(u[k][j], u[k][j]);
        group_sums_of<MIXED, K, V>(p, sum, bnorm_smem, buffer, turn);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            f2 w[P];
            params<V>(p.w_post, c[k], w);
            inverse_roots<MIXED, V>(sum[k], p.per_group, p.eps);
#pragma unroll
            for (int j = 0; j < P; ++j)
                u[k][j] = mul2(u[k][j], mul2(sum[k][j], w[j]));
        }
    }
    f2 square = both(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        f2 f[P];
        if (p.z) {
            widen(z[k], f);
#pragma unroll
            for (int j = 0; j < P; ++j)
                u[k][j] = mul2(u[k][j], silu2(f[j]));
        }
        if (p.scale) {
            params<V>(p.scale, c[k], f);
#pragma unroll
            for (int j = 0; j < P; ++j)
                u[k][j] = mul2(u[k][j], f[j]);
        }
        if (p.r) {
            widen(r[k], f);
#pragma unroll
            for (int j = 0; j < P; ++j)
                u[k][j] = add2(u[k][j], f[j]);
        }
        if (p.h && ok[k])
            store<T, V>(static_cast<T*>(p.h) + row * p.ldh + c[k], u[k]);
        if (ok[k]) {
#pragma unroll
            for (int j = 0; j < P; ++j)
                square = fma2(u[k][j], u[k][j], square);
        }
    }
    if (!p.w_pre)
        return;
    float all[1] = {sum_of(square)};
    row_sums<1>(all, buffer, turn);
    const f2 rms = both(rsqrtf(fmaf(all[0], p.per_row, p.eps)));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        f2 w[P];
        params<V>(p.w_pre, c[k], w);
#pragma unroll
        for (int j = 0; j < P; ++j)
            u[k][j] = mul2(u[k][j], mul2(rms, w[j]));
        if (ok[k])
            store<T, V>(static_cast<T*>(p.y) + row * p.ldy + c[k], u[k]);
    }
}

// Workers (a block, or a warp of one) take every workers-th row and keep their shares of the parameters' gradients in registers.
//
// Where a thread has one vector of each operand of a row, copies of the next rows' vectors into its own places of shared memory are under way (kAhead rows; no other thread looks at
// them), so that memory is at work while the sums of a row are waited for (8192 x 2048: 106 -> 88 us; pairs of floats 88 -> 81).  80 registers for vectors of up to four elements, for more
// blocks on an SM; eight do not fit there (81 -> 99 us, spilled).
template <typename T, int V, int K, int MIXED>
__global__ void __maxnreg__(K == 1 && V < 8 ? 80 : K < 4 || V == 8 ? 128 : 64) norm_grad_kernel(const NormDev p)
{
    constexpr bool RING = K == 1 && V > 1;
    constexpr int P = kPairs<V>;
    __shared__ float buffer[2 * kSlot];
    wait_for_previous();
    const int worker = blockIdx.x * blockDim.y + threadIdx.y, vectors = p.d / V;
    int turn = 0;
    bool in[K];
    int c[K];
    f2 s_post[K][P], s_scale[K][P], s_pre[K][P];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = k * blockDim.x + threadIdx.x;
        in[k] = at < vectors;
        c[k] = in[k] ? at * V : 0;
#pragma unroll
        for (int j = 0; j < P; ++j)
            s_post[k][j] = s_scale[k][j] = s_pre[k][j] = both(0.f);
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
        const float eps = here ? p.eps : 1.f;    // (a row behind the last, of zeros, has finite roots whatever eps is: it adds zeros to the parameters' gradients)
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
        f2 g[K][P];
#pragma unroll
        for (int k = 0; k < K; ++k)
            widen(dh[k], g[k]);
        if (p.w_pre) {
            f2 square = both(0.f), product = both(0.f);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                f2 a[P], b[P], w[P];
                widen(h[k], a);
                widen(dy[k], b);
                params<V>(p.w_pre, c[k], w);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    square = fma2(a[j], a[j], square);
                    product = fma2(a[j], mul2(w[j], b[j]), product);
                }
            }
            float sums[2] = {sum_of(square), sum_of(product)};
            row_sums<2>(sums, buffer, turn);
            const float rms = rsqrtf(fmaf(sums[0], p.per_row, eps));
            const f2 rms2 = both(rms), mean = both(-sums[1] * p.per_row * rms * rms);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                f2 a[P], b[P], w[P];
                widen(h[k], a);
                widen(dy[k], b);
                params<V>(p.w_pre, c[k], w);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    s_pre[k][j] = fma2(mul2(a[j], rms2), b[j], s_pre[k][j]);
                    g[k][j] = fma2(rms2, fma2(a[j], mean, mul2(w[j], b[j])), g[k][j]);
                }
            }
        }
        if (p.dr) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (in[k] && here)
                    store<T, V>(static_cast<T*>(p.dr) + row * p.lddr + c[k], g[k]);
        }
        f2 inverse[K][P];
        if (p.w_post) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                f2 a[P];
                widen(x[k], a);
#pragma unroll
                for (int j = 0; j < P; ++j)
                    inverse[k][j] = mul2(a[j], a[j]);
            }
            group_sums_of<MIXED, K, V>(p, inverse, area, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k)
                inverse_roots<MIXED, V>(inverse[k], p.per_group, eps);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            f2 u[P], w[P];
            widen(x[k], u);
            if (p.w_post) {
                params<V>(p.w_post, c[k], w);
#pragma unroll
                for (int j = 0; j < P; ++j)
                    u[j] = mul2(mul2(u[j], inverse[k][j]), w[j]);
            }
            f2 gate[P], slope[P];
            if (p.z) {
                f2 f[P];
                widen(z[k], f);
#pragma unroll
                for (int j = 0; j < P; ++j) {    // silu, and its slope q + f q (1 - q)
                    const f2 q = sigmoid2(f[j]);
                    gate[j] = mul2(f[j], q);
                    slope[j] = fma2(gate[j], fma2(q, both(-1.f), both(1.f)), q);
                }
            }
            if (p.scale) {
                params<V>(p.scale, c[k], w);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    s_scale[k][j] = fma2(g[k][j], p.z ? mul2(u[j], gate[j]) : u[j], s_scale[k][j]);
                    g[k][j] = mul2(g[k][j], w[j]);
                }
            }
            if (p.z) {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    slope[j] = mul2(slope[j], mul2(g[k][j], u[j]));
                    g[k][j] = mul2(g[k][j], gate[j]);
                }
                if (p.dz && in[k] && here)
                    store<T, V>(static_cast<T*>(p.dz) + row * p.lddz + c[k], slope);
            }
        }
        if (p.w_post) {
            f2 sum[K][P];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                f2 a[P], w[P];
                widen(x[k], a);
                params<V>(p.w_post, c[k], w);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    s_post[k][j] = fma2(g[k][j], mul2(a[j], inverse[k][j]), s_post[k][j]);
                    g[k][j] = mul2(g[k][j], w[j]);
                    sum[k][j] = mul2(a[j], g[k][j]);
                }
            }
            group_sums_of<MIXED, K, V>(p, sum, area, buffer, turn);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                f2 a[P];
                widen(x[k], a);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const f2 mean = mul2(mul2(sum[k][MIXED ? j : 0], both(-p.per_group)), mul2(inverse[k][j], inverse[k][j]));
                    g[k][j] = mul2(inverse[k][j], fma2(a[j], mean, g[k][j]));
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
                    keep<V>(to + c[k], s_post[k]);
                if (p.dscale)
                    keep<V>(to + p.d + c[k], s_scale[k]);
                if (p.dw_pre)
                    keep<V>(to + 2 * p.d + c[k], s_pre[k]);
            }
    }
}

// The workers' shares added up in their order: 32 channels to a block, kRuns runs of workers side by side (2368 workers of 128 channels: with eight runs 22 us).
constexpr int kRuns = 32;
static __global__ void __launch_bounds__(32 * kRuns) norm_sum_kernel(const NormDev p)
{
    wait_for_previous();
    __shared__ float s[kRuns][33];
    const int lane = threadIdx.x % 32, run = threadIdx.x / 32, which = blockIdx.y, c = blockIdx.x * 32 + lane;
    float* to = which == 0 ? p.dw_post : which == 1 ? p.dscale : p.dw_pre;
    if (!to)
        return;
    float sum = 0.f;
    if (c < p.d) {
        const float* from = p.parts + (long long)which * p.d + c;
        const int lo = (int)((long long)p.workers * run / kRuns), hi = (int)((long long)p.workers * (run + 1) / kRuns);
        for (int w = lo; w < hi; w += 16) {      // sixteen loads under way together
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                v[i] = load_if(from + (long long)(w + i) * 3 * p.d, w + i < hi);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                sum += v[i];
        }
    }
    s[run][lane] = sum;
    __syncthreads();
    sum = s[lane][run];                          // a warp for each channel
#pragma unroll
    for (int o = 16; o; o /= 2)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const int mine = blockIdx.x * 32 + run;
    if (lane == 0 && mine < p.d)
        to[mine] = sum;
}

} // namespace bnorm
} // namespace ttc
