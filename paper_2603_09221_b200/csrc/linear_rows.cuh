// The projections' kernels beside the large matrix products (linear_umma.cuh): few rows, sums of a split contraction, dZ and
// the bias gradient, copies that give rows the alignment TMA asks for.
#pragma once

#include "linear_umma.cuh"

namespace ttc {
namespace lin {

// ---- few rows -----------------------------------------------------------------------------------------------------------
//
// Up to 8 NT rows (tokens) against all of W: W is read once, which bounds it.  A block takes 16 MT rows of W and a part of
// the contraction (a cluster shares the parts out and adds them up over the shared memory of its blocks); its eight warps deal
// that out again.  Each lane loads 16 contiguous bytes of two rows of W for every 16, and of one row of x for every 8, which are
// the operands of two mma.sync.m16n8k16: the instruction does not mind which contraction index a slot stands for, as long as
// both operands agree, so nothing is rearranged.  8 rows, 2048 -> 4096: 4.6 us for 16.8 MB of W (one round of loads); 8192 -> 8192
// 28.9 us, 4.6 TB/s; 32 rows 9.3 and 33.7, of which L2 gives the blocks as many bytes of x as of W.

constexpr int kFewWarps = 8;

// Rows of W of a block (16 MT), loads of a lane for 32 contraction indices, and as many such steps as are under way together:
// in registers, or, where those hold too few of them, in shared memory (2048 -> 4096 and 8192 -> 8192: 8 rows 5.7 and 28.9 us by
// registers, 6.1 and 28.0 by shared memory; 16 rows 6.6 and 34.8, 7.0 and 32.0; 32 rows 9.9 and 40.1, 9.3 and 33.8).
template <int NT> struct FewShape {
    static constexpr int MT = NT <= 2 ? 1 : 2, COLS = 16 * MT, LOADS = 2 * MT + NT;
    static constexpr bool RING = NT > 2;
    static constexpr int DEPTH = RING ? 24 / LOADS : NT == 1 ? 8 : 4;
    static constexpr int SUMS = kFewWarps * NT * 8 * (COLS + 1) * 4, HELD = RING ? DEPTH * kFewWarps * LOADS * 32 * 16 : 0;
    static constexpr int SMEM = HELD > SUMS ? HELD : SUMS;
};

struct FewDev {
    const void *x, *w;
    long long ldx, ldw;
    int rows, k, m;
    int part;                    // contraction indices of a block, a multiple of 8 where there is more than one part
    int vec;                     // rows of x and W can be read by 16 bytes, and end on them
    Epilogue e;
};

template <typename T> __device__ __forceinline__ uint4 load8(const T* row, bool row_ok, int k, int k_end, bool vec)
{
    if (vec)                                                         // (k_end is a multiple of 8)
        return load_if(reinterpret_cast<const uint4*>(row + k), row_ok && k < k_end);
    const unsigned short* u = reinterpret_cast<const unsigned short*>(row);
    unsigned short v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = row_ok && k + i < k_end ? u[k + i] : 0;
    uint4 r;
    r.x = v[0] | (unsigned)v[1] << 16, r.y = v[2] | (unsigned)v[3] << 16;
    r.z = v[4] | (unsigned)v[5] << 16, r.w = v[6] | (unsigned)v[7] << 16;
    return r;
}

template <typename T> __device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<bf16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__half>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T, typename OT> __device__ __forceinline__ void finish(const Epilogue& e, long long row, long long col, float z)
{
    if (e.bias)
        z += e.bias[col];
    if (e.pre)
        static_cast<T*>(e.pre)[row * e.ldp + col] = from_f<T>(z);
    z = activate(z, e.act);
    if (e.residual)
        z += to_f(static_cast<const OT*>(e.residual)[row * e.ldr + col]);
    static_cast<OT*>(e.out)[row * e.ldo + col] = from_f<OT>(z);
}

template <typename T, typename OT, int NT>
__global__ void __launch_bounds__(kFewWarps * 32, 2) few_rows_kernel(const FewDev p)
{
    wait_for_previous();
    using S = FewShape<NT>;
    constexpr int MT = S::MT, COLS = S::COLS, LOADS = S::LOADS, DEPTH = S::DEPTH;
    extern __shared__ uint4 s_few[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int f0 = blockIdx.x * COLS, parts = gridDim.y;
    const int begin = blockIdx.y * p.part, end = min(p.k, begin + p.part);
    const T *w = static_cast<const T*>(p.w) + (long long)(f0 + g) * p.ldw, *x = static_cast<const T*>(p.x) + (long long)g * p.ldx;
    const long long w8 = 8 * p.ldw, x8 = 8 * p.ldx;
    const int steps = (end - begin - warp * 32 + kFewWarps * 32 - 1) / (kFewWarps * 32);           // (the same for all lanes: mma.sync is theirs together)
    auto index = [&](int step) { return begin + (step * kFewWarps + warp) * 32 + t * 8; };
    float acc[MT][NT][4] = {};
    auto multiply = [&](const uint4 (&a)[2 * MT], const uint4& b, int n) {
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            mma16816<T>(acc[j][n], a[2 * j].x, a[2 * j + 1].x, a[2 * j].y, a[2 * j + 1].y, b.x, b.y);
            mma16816<T>(acc[j][n], a[2 * j].z, a[2 * j + 1].z, a[2 * j].w, a[2 * j + 1].w, b.z, b.w);
        }
    };
    if constexpr (!S::RING) {
        for (int i0 = 0; i0 < steps; i0 += DEPTH) {
            uint4 a[DEPTH][2 * MT], b[DEPTH][NT];
#pragma unroll
            for (int i = 0; i < DEPTH; ++i) {
                const int k = index(i0 + i);
#pragma unroll
                for (int j = 0; j < 2 * MT; ++j)
                    a[i][j] = load8(w + j * w8, f0 + g + 8 * j < p.m, k, end, p.vec);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    b[i][n] = load8(x + n * x8, n * 8 + g < p.rows, k, end, p.vec);
            }
#pragma unroll
            for (int i = 0; i < DEPTH; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    multiply(a[i], b[i][n], n);
        }
    } else {
        // places in shared memory that only this lane writes and reads
        uint4* ring = s_few + warp * (LOADS * 32) + lane;
        auto copy = [&](uint4* to, const T* row, bool ok, int k) {
            if (p.vec) {
                const bool in = ok && k < end;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(smem_u32(to)), "l"(in ? row + k : static_cast<const T*>(p.w)), "r"(in ? 16 : 0) : "memory");
            } else {
                *to = load8(row, ok, k, end, false);
            }
        };
        auto fetch = [&](int step) {
            if (step < steps) {
                uint4* to = ring + step % DEPTH * (kFewWarps * LOADS * 32);
#pragma unroll
                for (int j = 0; j < 2 * MT; ++j)
                    copy(to + j * 32, w + j * w8, f0 + g + 8 * j < p.m, index(step));
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    copy(to + (2 * MT + n) * 32, x + n * x8, n * 8 + g < p.rows, index(step));
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < DEPTH; ++i)
            fetch(i);
        for (int i = 0; i < steps; ++i) {
            asm volatile("cp.async.wait_group %0;" :: "n"(DEPTH - 1) : "memory");
            const uint4* from = ring + i % DEPTH * (kFewWarps * LOADS * 32);
            uint4 a[2 * MT];
#pragma unroll
            for (int j = 0; j < 2 * MT; ++j)
                a[j] = from[j * 32];
#pragma unroll
            for (int n = 0; n < NT; ++n)
                multiply(a, from[(2 * MT + n) * 32], n);
            fetch(i + DEPTH);                                        // behind the products: what they read is overwritten
        }
    }
    __syncthreads();                                                 // (no copy is under way: the last groups are empty)
    float (*part)[NT * 8][COLS + 1] = reinterpret_cast<float (*)[NT * 8][COLS + 1]>(s_few);
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            part[warp][n * 8 + 2 * t][16 * j + g] = acc[j][n][0];
            part[warp][n * 8 + 2 * t + 1][16 * j + g] = acc[j][n][1];
            part[warp][n * 8 + 2 * t][16 * j + g + 8] = acc[j][n][2];
            part[warp][n * 8 + 2 * t + 1][16 * j + g + 8] = acc[j][n][3];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 8 * COLS; i += kFewWarps * 32) {
        const int row = i / COLS, f = i % COLS;
        float z = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWarps; ++k)
            z += part[k][row][f];
        if (parts > 1)
            part[0][row][f] = z;                                     // for the cluster
        else if (row < p.rows && f0 + f < p.m)
            finish<T, OT>(p.e, row, f0 + f, z);
    }
    if (parts == 1)
        return;
    __syncwarp();
    cluster_sync();
    for (int i = blockIdx.y * (kFewWarps * 32) + threadIdx.x; i < NT * 8 * COLS; i += parts * (kFewWarps * 32)) {
        const int row = i / COLS, f = i % COLS;
        if (row >= p.rows || f0 + f >= p.m)
            continue;
        const uint32_t at = smem_u32(&part[0][row][f]);
        float z = 0.f;
        for (int s = 0; s < parts; ++s) {
            uint32_t there;
            float v;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(s));
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
            z += v;
        }
        finish<T, OT>(p.e, row, f0 + f, z);
    }
    __syncwarp();
    cluster_sync();                                                  // no block ends while another one reads its sums
}

// ---- the parts of a split contraction ---------------------------------------------------------------------------------

template <typename T, typename OT>
__global__ void __launch_bounds__(256) split_sum_kernel(const float* part, long long split_stride, int splits, long long M, long long N, const Epilogue e)
{
    wait_for_previous();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= M * N)
        return;
    float z = 0.f;
    for (int s = 0; s < splits; ++s)
        z += part[s * split_stride + i];
    finish<T, OT>(e, i / N, i % N, z);
}

// ---- dZ and the sums over the rows --------------------------------------------------------------------------------------

template <int ACT> __device__ __forceinline__ float act_slope(float z)
{
    if (ACT == TTC_ACT_RELU)
        return z > 0.f ? 1.f : 0.f;
    if (ACT == TTC_ACT_SILU)
        return silu_slope(z);
    if (ACT == TTC_ACT_GELU) {
        float bell;
        const float cdf = normal_cdf(z, bell);
        return fmaf(z * 0.39894228040143268f, bell, cdf);
    }
    return ACT == TTC_ACT_SOFTPLUS ? sigmoid(z) : 1.f;
}

struct SlopeDev {
    long long rows;
    int m, rows_per_block;
    const void *dy, *pre;
    long long lddy, ldp;
    void* dz;                    // null: dy is used as it is
    long long lddz;
    float* part;                 // [blocks of rows][m] or null
};

// dZ = dy act'(pre) in 16 bits, and each block's sums over its rows, of the unrounded values.  V columns to a thread.  Bound by
// memory: 8192 x 8192 in bfloat16 with GELU 78 us for 403 MB, 5.2 TB/s.
template <typename T, typename OT, int V, int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const SlopeDev p)
{
    __shared__ float sums[8][32][V + 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int c = (blockIdx.x * 32 + lane) * V;
    const long long r0 = (long long)blockIdx.y * p.rows_per_block, r1 = min(p.rows, r0 + p.rows_per_block);
    float s[V] = {};
    if (c < p.m) {
        for (long long r = r0 + warp; r < r1; r += 8) {
            const Vec<OT, V> g = *reinterpret_cast<const Vec<OT, V>*>(static_cast<const OT*>(p.dy) + r * p.lddy + c);
            Vec<T, V> z, o;
            if (ACT != TTC_ACT_NONE)
                z = *reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.pre) + r * p.ldp + c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float d = to_f(g.v[i]);
                if (ACT != TTC_ACT_NONE)
                    d = __fmul_rn(d, act_slope<ACT>(to_f(z.v[i])));  // (never one operation with the sum: dbias has the same bits with and without dZ)
                s[i] += d;
                o.v[i] = from_f<T>(d);
            }
            if (p.dz)
                *reinterpret_cast<Vec<T, V>*>(static_cast<T*>(p.dz) + r * p.lddz + c) = o;
        }
    }
    if (!p.part)
        return;
#pragma unroll
    for (int i = 0; i < V; ++i)
        sums[warp][lane][i] = s[i];
    __syncthreads();
    for (int at = threadIdx.x; at < 32 * V; at += 256) {
        const int l = at / V, i = at % V, col = (blockIdx.x * 32 + l) * V + i;
        if (col >= p.m)
            continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w)
            v += sums[w][l][i];
        p.part[(long long)blockIdx.y * p.m + col] = v;
    }
}

static __global__ void __launch_bounds__(256) bias_sum_kernel(const float* part, int blocks, int m, float* out)
{
    wait_for_previous();
    __shared__ float sum[8][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < m)
        for (int b = warp; b < blocks; b += 8)
            s += part[(long long)b * m + c];
    sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < m) {
        for (int k = 1; k < 8; ++k)
            s += sum[k][lane];
        out[c] = s;
    }
}

// Rows copied to a stride that is a multiple of 16 bytes.
static __global__ void __launch_bounds__(256) align_rows_kernel(const unsigned short* from, long long ld, long long rows, int cols, unsigned short* to, long long ldt)
{
    wait_for_previous();
    const long long r = blockIdx.x;
    for (int c = threadIdx.x; c < cols; c += 256)
        to[r * ldt + c] = from[r * ld + c];
}

template <typename T> __global__ void __launch_bounds__(256) zero_rows_kernel(T* to, long long ld, long long rows, int cols)
{
    wait_for_previous();
    for (int c = threadIdx.x; c < cols; c += 256)
        to[(long long)blockIdx.x * ld + c] = from_f<T>(0.f);
}

} // namespace lin
} // namespace ttc
