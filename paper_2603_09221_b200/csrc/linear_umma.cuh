// Matrix products of the projections on the 5th-generation tensor cores: D[i][j] = sum_k A(i, k) B(j, k), with what is to
// be done to a product before it is written (bias, activation, residual) done on the accumulators.
//
// One CTA per SM works through tiles of 128 x BN, or, where there are enough of them, two neighbouring ones through tiles of
// 256 x 256 (cta_group::2): each then fetches and reads 64 KB of shared memory for a block of 64 contraction indices instead
// of 96, which is what bounds a single CTA (128 bytes per clock: 768 clocks against 512 of products).  One warp keeps a ring of
// stages of 64 contraction indices filled by TMA (128-byte swizzle), one issues tcgen05.mma (kind::f16) into one of two
// accumulators in tensor memory, and eight warps read the other one back, so that the end of a tile runs beside the products
// of the next.  Operands are read as they lie in memory: an operand whose contraction index is not the contiguous one (the
// gradients') is staged in boxes of 64 contiguous rows by 64 contraction indices and described to the instruction as MN-major;
// nothing is transposed.  Rows, columns and contraction indices past the end are filled with zeros by TMA.
//
// bfloat16, 8192 x 8192 over 8192: 692 to 738 us by the clock, 1589 TFLOP/s (torch.mm in the same loops 682 to 787); 8192 x 2048 over 4096 93 us alone
// and 97 back to back (92, 94), where power bounds both.  512 x 4096 over 2048 13.7 us (9.9): one round of tiles, whose start and end
// nothing hides.  Float32 results with softplus, 4096 x 2304 over 1024: 26.8 us, of which the end of a tile, 9 us, comes twice.
// Sums in segments: 4096 x 2048 over 2048 36 us (30 without).
#pragma once

#include <cuda.h>

#include "block_common.cuh"

namespace ttc {
namespace lin {

using namespace blk;

constexpr int BM = 128, BK = 64;
constexpr int kEpilogueWarps = 8;
constexpr int kGemmThreads = 32 * (2 + kEpilogueWarps);
constexpr int kSpinLimit = 1 << 22;
constexpr int kStageRow = 80;                    // bytes of a staged row of 64, padded against bank conflicts

static __device__ int g_error;                   // set where a wait gave up

struct Epilogue {
    void* out;                   // [M][N], or [splits][M][N] floats of a split contraction
    long long ldo, split_stride;
    const float* bias;           // [N] or null
    const void* residual;        // type of out, or null
    long long ldr;
    void* pre;                   // z in 16 bits, or null
    long long ldp;
    int act, pre_bf16;
    int vec_o, vec_r, vec_p;     // rows can be accessed by 16 bytes
};

struct GemmDev {
    long long M, N;
    int k_blocks;                // blocks of BK contraction indices in all
    int splits;                  // parts of the contraction, each a tile of its own
    int segment;                 // float32 results: blocks of BK that the tensor cores add up before the sum goes to registers
    int tiles_m, tiles_n;
    uint32_t idesc;
    Epilogue e;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Gives up after kSpinLimit polls, or once another thread of the CTA has; then the CTA stops.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* dead)
{
    for (int i = 0; i < kSpinLimit; ++i) {
        if (try_wait(bar, parity))
            return true;
        if ((i & 63) == 63 && *dead)
            return false;
    }
    *dead = 1;
    g_error = 1;
    return false;
}
// true in one lane of the (converged) warp
__device__ __forceinline__ bool elect_one()
{
    uint32_t pred;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(pred));
    return pred != 0;
}
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity)
{
    for (int i = 0; i < kSpinLimit && !try_wait(bar, parity); ++i) {
    }
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// ---- two CTAs of a cluster on one tile (cta_group::2) ----
// The same barrier of the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(uint32_t bar)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" :: "r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t at, float (&v)[32])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i)
        v[i] = __uint_as_float(r[i]);
}
// eight columns added to v
__device__ __forceinline__ void tmem_add8(uint32_t at, float* v)
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] += __uint_as_float(r[i]);
}

// Shared-memory descriptors (128-byte swizzle).  K-major: rows of 64 contraction indices, 128 bytes each, groups of eight
// rows 1024 bytes apart; a step of 16 indices is 32 bytes further in.  MN-major: rows of 64 indices of the other dimension, one
// for each contraction index, groups of eight 1024 bytes apart; the next 64 are a box (8192 bytes) further; a step of 16
// contraction indices is 2048 bytes.
template <bool MN> __device__ __forceinline__ uint64_t operand_desc(uint32_t at)
{
    const uint64_t lead = MN ? (8192 >> 4) : 1;
    return (uint64_t)((at >> 4) & 0x3fffu) | lead << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// Instruction descriptor: float32 accumulators, both operands bfloat16 or both float16.
inline uint32_t instruction(bool is_bf16, bool a_mn, bool b_mn, int bm, int bn)
{
    const uint32_t f = is_bf16 ? 1 : 0;
    return 1u << 4 | f << 7 | f << 10 | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 | (uint32_t)(bn >> 3) << 17 | (uint32_t)(bm >> 4) << 24;
}

// Activations of 32 results; the choice lies outside of the loop.
template <typename F> __device__ __forceinline__ void each(float (&v)[32], F&& f)
{
#pragma unroll
    for (int i = 0; i < 32; ++i)
        v[i] = f(v[i]);
}
template <typename F> __device__ __forceinline__ void each_pair(float (&v)[32], F&& f)
{
#pragma unroll
    for (int i = 0; i < 32; i += 2)
        unpack2(f(pack2(v[i], v[i + 1])), v[i], v[i + 1]);
}
__device__ __forceinline__ float activate(float z, int act)
{
    switch (act) {
    case TTC_ACT_RELU: return z < 0.f ? 0.f : z;                                   // NaN stays NaN
    case TTC_ACT_SILU: return silu(z);
    case TTC_ACT_GELU: return gelu(z);
    case TTC_ACT_SOFTPLUS: return softplus(z);
    default: return z;
    }
}
__device__ __forceinline__ void activate(float (&v)[32], int act)
{
    switch (act) {
    case TTC_ACT_RELU: return each(v, [](float z) { return activate(z, TTC_ACT_RELU); });
    case TTC_ACT_SILU: return each_pair(v, [](f2 z) { return silu2(z); });
    case TTC_ACT_GELU: return each(v, [](float z) { return activate(z, TTC_ACT_GELU); });
    case TTC_ACT_SOFTPLUS: return each_pair(v, [](f2 z) { return softplus2(z); });
    default: return;
    }
}

template <typename OT> __device__ __forceinline__ void load_chunk(const OT* at, bool row_ok, long long cols, bool vec, float (&v)[32])
{
    constexpr int V = 16 / sizeof(OT);
    if (!row_ok) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            v[i] = 0.f;
    } else if (vec && cols >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += V) {
            const Vec<OT, V> u = *reinterpret_cast<const Vec<OT, V>*>(at + i);
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[i + j] = to_f(u.v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            v[i] = i < cols ? to_f(at[i]) : 0.f;
    }
}

// Writes 32 rows x 32 columns, a row in each lane, through the warp's staging rows: rows of 64 bytes leave in 16-byte pieces.
template <typename OT>
__device__ __forceinline__ void store_chunk(const float (&v)[32], OT* at, long long ld, long long rows, long long cols, bool vec, char* stage, int lane)
{
    constexpr int V = 16 / sizeof(OT), C = 64 / sizeof(OT);          // columns of a 64-byte row
#pragma unroll
    for (int c0 = 0; c0 < 32; c0 += C) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < C; i += V) {
            Vec<OT, V> u;
#pragma unroll
            for (int j = 0; j < V; ++j)
                u.v[j] = from_f<OT>(v[c0 + i + j]);
            *reinterpret_cast<Vec<OT, V>*>(stage + lane * kStageRow + i * sizeof(OT)) = u;
        }
        __syncwarp();
        if (vec && cols >= c0 + C) {
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 8) {
                const int r = r0 + lane / 4, part = lane % 4;
                if (r < rows)
                    *reinterpret_cast<uint4*>(at + r * ld + c0 + part * V) = *reinterpret_cast<const uint4*>(stage + r * kStageRow + part * 16);
            }
        } else {
            for (int e = lane; e < 32 * C; e += 32) {
                const int r = e / C, c = e % C;
                if (r < rows && c0 + c < cols)
                    at[r * ld + c0 + c] = *reinterpret_cast<const OT*>(stage + r * kStageRow + c * sizeof(OT));
            }
        }
    }
}

// PAIR: two CTAs on a tile of 256 x BN, each with half of the rows of either operand and half of the results.
template <int BN, bool PAIR> struct GemmShape {
    static constexpr int B_ROWS = PAIR ? BN / 2 : BN;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = B_ROWS * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int STAGES = 196608 / STAGE_BYTES;
    static constexpr int EPI_BYTES = kEpilogueWarps * (32 * kStageRow + 128 * 4);
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + EPI_BYTES + 256;
};

// SEGMENTS: the tensor cores cut sums off instead of rounding them, an error that grows with the contraction (1.0e-6 of the
// result's norm at 1024 indices); the results of longer ones are then added up in registers, segment by segment.
template <bool A_MN, bool B_MN, int BN, bool PAIR, typename OT, bool SEGMENTS>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                              const GemmDev p)
{
    using S = GemmShape<BN, PAIR>;
    constexpr int STAGES = S::STAGES, CTAS = PAIR ? 2 : 1;
    extern __shared__ char smem_raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) / 1024 * 1024);
    char* s_epi = smem + STAGES * S::STAGE_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_epi + S::EPI_BYTES);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, acc_full = empty + 8 * STAGES, acc_empty = acc_full + 16,
                   drained = acc_empty + 16;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 5);
    volatile int* dead = reinterpret_cast<volatile int*>(s_tmem + 1);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int rank = PAIR ? blockIdx.x % 2 : 0;                      // in the cluster
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * STAGES; ++i)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(full + 8 * i) : "memory");
        for (int i = 0; i < 2; ++i) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(acc_full + 8 * i) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(acc_empty + 8 * i), "r"(CTAS * kEpilogueWarps) : "memory");
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(drained) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        *dead = 0;
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(s_tmem)), "r"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(s_tmem)), "r"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    __syncwarp();
    if (PAIR)
        cluster_sync();                                              // the other CTA's barriers and tensor memory are there
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, *s_tmem, 0);
    wait_for_previous();                                             // what stands above needs nothing of it

    const int per_split = p.tiles_m * p.tiles_n, tiles = per_split * p.splits;
    // Tiles of eight rows of tiles follow one another column by column, so that the CTAs at work share operands in L2.
    auto place = [&](int tile, int& mt, int& nt, int& k0, int& k1) {
        const int split = tile / per_split, at = tile % per_split;
        const int band = at / (8 * p.tiles_n), height = min(8, p.tiles_m - band * 8), in = at - band * 8 * p.tiles_n;
        mt = band * 8 + in % height;
        nt = in / height;
        k0 = static_cast<int>((long long)p.k_blocks * split / p.splits);
        k1 = static_cast<int>((long long)p.k_blocks * (split + 1) / p.splits);
        return split;
    };

    const int first_tile = blockIdx.x / CTAS, tile_step = gridDim.x / CTAS;
    // Both issuing warps walk their loops as a whole and elect a lane for the instruction itself: what it is given then comes
    // from uniform registers (from one lane's own registers the products of a stage took 500 clocks to issue).
    const uint32_t stages = __shfl_sync(0xffffffffu, smem_u32(smem), 0);
    if (warp == 0) {
        unsigned it = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            int mt, nt, k0, k1;
            place(tile, mt, nt, k0, k1);
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % STAGES;
                if (!(ok = wait(empty + 8 * s, (it / STAGES & 1) ^ 1, dead)))
                    break;
                const uint32_t bar = full + 8 * s, a = stages + s * S::STAGE_BYTES, b = a + S::A_BYTES;
                // rows of the operands that this CTA fetches; a pair's copies all count on the first CTA's barrier
                const int ra = (mt * CTAS + rank) * BM, rb = nt * BN + rank * S::B_ROWS;
                const uint32_t counted = PAIR ? in_first(bar) : bar;
                auto fetch = [&](uint32_t to, const CUtensorMap* map, int x, int y) {
                    if (PAIR)
                        tma_load_pair(to, map, x, y, counted);
                    else
                        tma_load(to, map, x, y, counted);
                };
                if (elect_one()) {
                    if (rank == 0)
                        expect_bytes(bar, CTAS * S::STAGE_BYTES);
                    if (A_MN) {
#pragma unroll
                        for (int i = 0; i < BM / 64; ++i)
                            fetch(a + i * 8192, &map_a, ra + i * 64, k * BK);
                    } else {
                        fetch(a, &map_a, k * BK, ra);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int i = 0; i < S::B_ROWS / 64; ++i)
                            fetch(b + i * 8192, &map_b, rb + i * 64, k * BK);
                    } else {
                        fetch(b, &map_b, k * BK, rb);
                    }
                }
                __syncwarp();
            }
        }
        if (!ok) {                                                   // copies under way end before the CTA does
            if (rank == 0) {
                for (unsigned i = it > STAGES ? it - STAGES : 0; i < it; ++i)
                    drain(full + 8 * (i % STAGES), i / STAGES & 1);
            } else {                                                 // theirs count on a barrier that only the first CTA can look at
                for (int i = 0; i < 1000; ++i)
                    __nanosleep(1000);
            }
        }
    } else if (warp == 1 && rank == 0) {
        unsigned it = 0, done = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            int mt, nt, begin, end;
            place(tile, mt, nt, begin, end);
            for (int k0 = begin; ok && k0 < end; ++done) {
                const int k1 = SEGMENTS ? min(end, k0 + p.segment) : end;
                const uint32_t d = tmem + (done & 1) * BN;
                if (!(ok = wait(acc_empty + 8 * (done & 1), (done / 2 & 1) ^ 1, dead)))
                    break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int k = k0; k < k1; ++k, ++it) {
                    const int s = it % STAGES;
                    if (!(ok = wait(full + 8 * s, it / STAGES & 1, dead)))
                        break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t a = stages + s * S::STAGE_BYTES, b = a + S::A_BYTES;
                    const uint64_t da = operand_desc<A_MN>(a), db = operand_desc<B_MN>(b);
                    if (elect_one()) {
#pragma unroll
                        for (int j = 0; j < BK / 16; ++j)
                            if (PAIR)
                                mma_pair(d, da + j * ((A_MN ? 2048 : 32) >> 4), db + j * ((B_MN ? 2048 : 32) >> 4), p.idesc, k > k0 || j > 0);
                            else
                                mma(d, da + j * ((A_MN ? 2048 : 32) >> 4), db + j * ((B_MN ? 2048 : 32) >> 4), p.idesc, k > k0 || j > 0);
                        if (PAIR) {
                            commit_pair(empty + 8 * s);
                            if (k + 1 == k1)
                                commit_pair(acc_full + 8 * (done & 1));
                        } else {
                            commit(empty + 8 * s);
                            if (k + 1 == k1)
                                commit(acc_full + 8 * (done & 1));
                        }
                    }
                    __syncwarp();
                }
                k0 = k1;
            }
        }
        if (!ok) {                                                   // products under way end before tensor memory is given back
            if (elect_one()) {
                if (PAIR)
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(drained) : "memory");
                else
                    commit(drained);
            }
            __syncwarp();
            drain(drained, 0);
        }
    } else if (warp >= 2) {
        const int w = warp - 2, quarter = warp % 4, half = w / 4;    // a warp reads the lanes of its quarter of tensor memory
        char* stage = s_epi + w * (32 * kStageRow + 128 * 4);
        float* s_bias = reinterpret_cast<float*>(stage + 32 * kStageRow);
        unsigned done = 0;
        for (int tile = first_tile; tile < tiles; tile += tile_step, done += SEGMENTS ? 0 : 1) {
            int mt, nt, k0, k1;
            const int split = place(tile, mt, nt, k0, k1);
            const long long row0 = ((long long)mt * CTAS + rank) * BM + quarter * 32, col0 = (long long)nt * BN + half * (BN / 2);
            __syncwarp();
            for (int c = lane; c < BN / 2; c += 32)
                s_bias[c] = p.e.bias && col0 + c < p.N ? p.e.bias[col0 + c] : 0.f;
            __syncwarp();
            bool ok = true;
            float sum[SEGMENTS ? BN / 64 : 1][32] = {};
            if (SEGMENTS) {
                for (int k = k0; ok && k < k1; k += p.segment, ++done) {
                    if (!(ok = wait(acc_full + 8 * (done & 1), done / 2 & 1, dead)))
                        break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t from = tmem + (done & 1) * BN + half * (BN / 2) + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 8)
                        tmem_add8(from + c, &sum[SEGMENTS ? c / 32 : 0][c % 32]);
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR)
                            arrive_cluster(in_first(acc_empty + 8 * (done & 1)));
                        else
                            arrive(acc_empty + 8 * (done & 1));
                    }
                }
            } else {
                ok = wait(acc_full + 8 * (done & 1), done / 2 & 1, dead);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            if (!ok)
                break;
            const uint32_t from = tmem + (done & 1) * BN + half * (BN / 2) + ((uint32_t)(quarter * 32) << 16);
            OT* out = static_cast<OT*>(p.e.out) + split * p.e.split_stride;
#pragma unroll(SEGMENTS ? BN / 64 : 1)
            for (int c = 0; c < BN / 2; c += 32) {
                float v[32];
                if (SEGMENTS) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        v[i] = sum[SEGMENTS ? c / 32 : 0][i];
                } else {
                    tmem_ld32(from + c, v);
                }
                if (!SEGMENTS && c + 32 == BN / 2) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR)
                            arrive_cluster(in_first(acc_empty + 8 * (done & 1)));
                        else
                            arrive(acc_empty + 8 * (done & 1));
                    }
                }
                const long long rows = p.M - row0, cols = p.N - (col0 + c);
                if (rows <= 0 || cols <= 0)
                    continue;
                if (p.e.bias) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 b = *reinterpret_cast<const float4*>(s_bias + c + i);
                        v[i] += b.x, v[i + 1] += b.y, v[i + 2] += b.z, v[i + 3] += b.w;
                    }
                }
                if (p.e.pre) {
                    if (p.e.pre_bf16)
                        store_chunk(v, static_cast<bf16*>(p.e.pre) + row0 * p.e.ldp + col0 + c, p.e.ldp, rows, cols, p.e.vec_p, stage, lane);
                    else
                        store_chunk(v, static_cast<__half*>(p.e.pre) + row0 * p.e.ldp + col0 + c, p.e.ldp, rows, cols, p.e.vec_p, stage, lane);
                }
                activate(v, p.e.act);
                if (p.e.residual) {
                    float r[32];
                    load_chunk(static_cast<const OT*>(p.e.residual) + (row0 + lane) * p.e.ldr + col0 + c, lane < rows, cols, p.e.vec_r, r);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        v[i] += r[i];
                }
                store_chunk(v, out + row0 * p.e.ldo + col0 + c, p.e.ldo, rows, cols, p.e.vec_o, stage, lane);
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    __syncwarp();
    if (PAIR)
        cluster_sync();                                              // neither CTA is signalled after it has ended
    if (warp == 1) {
        if (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(2 * BN) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(2 * BN) : "memory");
    }
}

} // namespace lin
} // namespace ttc
