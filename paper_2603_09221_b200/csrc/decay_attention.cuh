// Linear attention with a decay for each head:  S_t = exp(l_t) S_{t-1} + k_t v_t',  y_t = scale q_t S_t,  l_t = A D_t.
//
// Token by token this is 5 dk dv operations on a state that no register file holds.  Over a chunk of 128 tokens, with
// G_i = l_1 + .. + l_i from the chunk's first token and R_j = l_{j+1} + .. + l_128, it is
//
//     y_i = scale [ sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j  +  exp(G_i) q_i S_0 ],      S_C = exp(G_C) S_0 + sum_j exp(R_j) k_j v_j'
//
// four products of 128 rows each, which the 5th-generation tensor cores take, and the chunks depend on one another through S only:
//
//     chunk_state_kernel   U = sum_j exp(R_j) k_j v_j' of every chunk and head
//     state_scan_kernel    S_0 of every chunk from S_C = exp(G_C) S_0 + U, element by element
//     chunk_out_kernel     y
//
// Exponents.  None is positive: pairs of tokens of one block of 32 take exp(G_i - G_j) itself, from sums within the block; others the product
// of exp(from the block's begin to i) and exp(from j to that begin), so that no difference of long sums is formed.  Exponents
// below -192 / log2(e) count as that (their exponentials are zero), so that a decay of minus infinity, which forgets
// everything, gives no difference of infinities.
//
// Roundings.  Sums are float32 in tensor memory, states float32.  Operands of the tensor cores are 16 bits: scores with their decay, and S_0 where q
// multiplies it, are rounded once (half a step each, as the result itself).  The weighted keys of U are not: states are float32 results and are carried on, so
// the keys go in as a sum of numbers of 16 bits, each what the ones before it left: three bfloat16 or two float16 (2^-24, 2^-22 of the value; two bfloat16 leave 2^-18,
// and the states were off by 2.4e-6 in the 2-norm).
#pragma once

#include <type_traits>

#include "pieces.cuh"
#include "umma.cuh"

namespace ttc {
namespace dattn {

using namespace blk;
using namespace umma;

constexpr int kChunk = 128;
constexpr int kThreads = 256;
constexpr float kFloor = -192.f;                 // of exponents to the base 2: 2^-192 is zero

struct AttnDev {
    Seqs seqs;
    const int2* piece_map;                       // packed sequences: sequence and first token of each chunk
    const int* seq_first;                        // and the first chunk of each sequence
    long long chunks_per_seq, chunks;            // equal sequences; chunks in all (packed: room for them)
    int heads, share, dk, dv;                    // share: heads of a group
    int softplus;
    float scale;
    Rows q, k, v, delta, y;
    int vec_q, vec_k, vec_v, vec_y;              // rows can be accessed by 16 bytes
    int vec_state;                               // and the states
    const float *A, *delta_bias, *state;
    float* state_out;
    // scratch
    float* added;                                // U: [chunks][heads][DV / 4][DK][4]
    float* whole;                                // exp(G_C): [chunks][heads]
    float* most;                                 // largest |U|: [chunks][heads] (float16)
    float* most_given;                           // and of the states that are given: [batch][heads] (float16)
    float* unit;                                 // what the image of S_0 has to be multiplied by: [chunks][heads] (float16)
    char* image;                                 // S_0 in 16 bits: [chunks][heads][1 or 2][DV / 8][DK][8]
};

struct Chunk {
    long long seq, row0;                         // sequence and row of the first token, as row_ptr takes them
    long long owner;                             // the sequence, where the chunk is its first one, else -1
    int len;                                     // tokens, 0: nothing to do
};

__device__ __forceinline__ Chunk chunk_at(const AttnDev& p, long long c)
{
    Chunk r;
    if (p.piece_map) {
        const int2 m = p.piece_map[c];
        if (m.x < 0)
            return Chunk{0, 0, -1, 0};
        const Span s = span_of(p.seqs, m.x);
        r.seq = 0;
        r.row0 = s.row0 + m.y;
        r.owner = m.y ? -1 : m.x;
        r.len = (int)min(s.len - m.y, (long long)kChunk);
    } else {
        r.seq = c / p.chunks_per_seq;
        r.row0 = (c % p.chunks_per_seq) * kChunk;
        r.owner = r.row0 ? -1 : r.seq;
        r.len = (int)min(p.seqs.tokens - r.row0, (long long)kChunk);
    }
    return r;
}

// ---- decays of a chunk --------------------------------------------------------------------------------------------------

struct alignas(16) Decays {
    float g[kChunk];                             // sums to the base 2 from the begin of the token's block of 32, the token's own included
    float s[kChunk];                             // behind the token, to the end of its block
    float block[4];                              // of whole blocks
};

__device__ __forceinline__ float step_of(const AttnDev& p, float raw) { return p.softplus ? softplus(raw) : raw; }

// What softplus or nothing is taken of, and the step; raw only where there is a delta.
template <typename T> __device__ __forceinline__ float raw_step(const AttnDev& p, long long seq, long long row, int head)
{
    return to_f(row_ptr<T>(p.delta, seq, row)[head]) + (p.delta_bias ? p.delta_bias[head] : 0.f);
}

template <typename T> __device__ __forceinline__ float log_decay(const AttnDev& p, const Chunk& c, int head, int t)
{
    if (t >= c.len)
        return 0.f;
    const float d = p.delta.ptr ? step_of(p, raw_step<T>(p, c.seq, c.row0 + t, head)) : 1.f;
    const float l = p.A[head] * d * kLog2e;
    return l < kFloor ? kFloor : l;              // NaN stays
}

// By the first four warps.
template <typename T> __device__ __forceinline__ void find_decays(const AttnDev& p, const Chunk& c, int head, Decays& o)
{
    const int t = threadIdx.x, lane = t % 32;
    const float l = log_decay<T>(p, c, head, t);
    float g = l, s = l;
#pragma unroll
    for (int i = 1; i < 32; i *= 2) {
        const float a = __shfl_up_sync(0xffffffffu, g, i), b = __shfl_down_sync(0xffffffffu, s, i);
        g += lane >= i ? a : 0.f;
        s += lane + i < 32 ? b : 0.f;
    }
    const float behind = __shfl_down_sync(0xffffffffu, s, 1);
    o.g[t] = g;
    o.s[t] = lane < 31 ? behind : 0.f;
    if (lane == 31)
        o.block[t / 32] = g;
}

// exp of the sum from the chunk's begin to token t, and from behind t to the chunk's end
__device__ __forceinline__ float from_begin(const Decays& d, int t)
{
    float e = d.g[t];
    for (int b = 0; b < t / 32; ++b)
        e += d.block[b];
    return ex2(e);
}
__device__ __forceinline__ float to_end(const Decays& d, int t)
{
    float e = d.s[t];
    for (int b = t / 32 + 1; b < 4; ++b)
        e += d.block[b];
    return ex2(e);
}
__device__ __forceinline__ float over_chunk(const Decays& d) { return ex2((d.block[0] + d.block[1]) + (d.block[2] + d.block[3])); }
// from behind token t of an earlier block to the begin of block b
__device__ __forceinline__ float to_block(const Decays& d, int t, int b)
{
    float e = d.s[t];
    for (int i = t / 32 + 1; i < b; ++i)
        e += d.block[i];
    return ex2(e);
}

// ---- tiles in shared memory -----------------------------------------------------------------------------------------------

// A tile of 128 tokens: boxes of 64 columns, rows of 128 bytes under the 128-byte swizzle, zeros behind the chunk's tokens and the head's channels.
constexpr int kBox = kChunk * 128;

__device__ __forceinline__ uint32_t tile_at(int row, int c8) { return (uint32_t)((c8 / 8) * kBox + row * 128 + (((c8 % 8) ^ (row & 7)) << 4)); }

__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool ok)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }
// what threads have written becomes visible to the tensor cores (before the barrier that they are issued behind)
__device__ __forceinline__ void to_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Thread t sees to the vectors t, t + 256, ..: the same ones wherever a tile is gone through.
template <typename T, int COLS> __device__ __forceinline__ void load_tile(uint32_t to, const Rows& r, const Chunk& c, int head, int width, bool vec)
{
    const T* base = row_ptr<T>(r, c.seq, c.row0) + (long long)head * width;
    if (vec) {
#pragma unroll
        for (int i = 0; i < kChunk * COLS / 8; i += kThreads) {
            const int e = i + threadIdx.x, row = e / (COLS / 8), c8 = e % (COLS / 8);
            const bool ok = row < c.len && c8 * 8 < width;
            copy16(to + tile_at(row, c8), ok ? base + row * r.ts + c8 * 8 : base, ok);
        }
    } else {
        for (int e = threadIdx.x; e < kChunk * COLS / 8; e += kThreads) {
            const int row = e / (COLS / 8), c8 = e % (COLS / 8);
            Vec<T, 8> u;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                u.v[j] = row < c.len && c8 * 8 + j < width ? base[row * r.ts + c8 * 8 + j] : from_f<T>(0.f);
            const uint4 w = *reinterpret_cast<const uint4*>(&u);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(to + tile_at(row, c8)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
        }
    }
}

// The tile of results staged in shared memory, to its rows.
template <typename T, int COLS> __device__ __forceinline__ void store_tile(const char* from, const Rows& r, const Chunk& c, int head, int width, bool vec)
{
    T* base = row_ptr<T>(r, c.seq, c.row0) + (long long)head * width;
    for (int e = threadIdx.x; e < kChunk * COLS / 8; e += kThreads) {
        const int row = e / (COLS / 8), c8 = e % (COLS / 8);
        if (row >= c.len || c8 * 8 >= width)
            continue;
        const uint4 w = *reinterpret_cast<const uint4*>(from + tile_at(row, c8));
        T* at = base + row * r.ts + c8 * 8;
        if (vec) {
            *reinterpret_cast<uint4*>(at) = w;
        } else {
            const Vec<T, 8> u = *reinterpret_cast<const Vec<T, 8>*>(&w);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c8 * 8 + j < width)
                    at[j] = u.v[j];
        }
    }
}

// Descriptors.  Of a tile: contraction over its columns (K-major; 16 of them are 32 bytes, 64 a box), or over its tokens (MN-major; 16 of them 2048 bytes).
__device__ __forceinline__ uint64_t desc(uint32_t at, uint32_t lead, uint32_t stride, uint64_t layout)
{
    return (uint64_t)((at >> 4) & 0x3fffu) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | (uint64_t)1 << 46 | layout << 61;
}
__device__ __forceinline__ uint64_t over_columns(uint32_t tile, int step) { return desc(tile + (step / 4) * kBox + (step % 4) * 32, 16, 1024, 2); }
__device__ __forceinline__ uint64_t over_tokens(uint32_t tile, int step) { return desc(tile + step * 2048, kBox, 1024, 2); }
// Of the image of a state, [DV / 8][DK rows][8]: 8 rows x 16 bytes lie together (no swizzle), as the threads of the scan write them.
template <int DK> __device__ __forceinline__ uint64_t image_over_dv(uint32_t image, int step) { return desc(image + step * 2 * DK * 16, DK * 16, 128, 0); }
template <int DK> __device__ __forceinline__ uint64_t image_over_dk(uint32_t image, int step) { return desc(image + step * 256, 128, DK * 16, 0); }

__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                    "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const float (&v)[32])
{
    uint32_t r[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            r[i] = __float_as_uint(v[h * 16 + i]);
        tmem_st16(at + h * 16, r);
    }
}
__device__ __forceinline__ void tmem_st_done() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void before_barrier() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void behind_barrier() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

template <typename T> __device__ __forceinline__ uint32_t pack16(float a, float b);
template <> __device__ __forceinline__ uint32_t pack16<bf16>(float a, float b)
{
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint32_t pack16<__half>(float a, float b)
{
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <typename T> __device__ __forceinline__ float2 unpack16(uint32_t v);
template <> __device__ __forceinline__ float2 unpack16<bf16>(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
template <> __device__ __forceinline__ float2 unpack16<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

template <typename T> constexpr bool kIsBf16 = std::is_same<T, bf16>::value;

// Barriers and tensor memory of a block.
struct Control {
    uint64_t bar[4];
    uint32_t tmem;
    int dead;
};

__device__ __forceinline__ uint32_t set_up(Control& c, int columns)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(smem_u32(&c.bar[i])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        c.dead = 0;
    }
    if (threadIdx.x / 32 == 4) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&c.tmem)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    before_barrier();
    __syncthreads();
    behind_barrier();
    return __shfl_sync(0xffffffffu, c.tmem, 0);
}
__device__ __forceinline__ void give_back(uint32_t tmem, int columns)
{
    before_barrier();
    __syncthreads();
    if (threadIdx.x / 32 == 4)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(columns) : "memory");
}
// Products are waited for by everybody; where that takes too long, everybody goes on (the error is noted), so that barriers stay in step.
__device__ __forceinline__ void products_done(Control& c, int i, uint32_t parity = 0)
{
    wait(smem_u32(&c.bar[i]), parity, &c.dead);
    __syncwarp();
    behind_barrier();
}

extern __shared__ char dattn_smem[];
__device__ __forceinline__ char* aligned_smem() { return reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(dattn_smem) + 1023) / 1024 * 1024); }

// ---- what a chunk adds to the state ---------------------------------------------------------------------------------------

template <typename T, int DK, int DV> struct StateShape {
    static constexpr int TERMS = kIsBf16<T> ? 3 : 2;                 // numbers of 16 bits that a weighted key is split into
    static constexpr int A_BYTES = DK / 64 * kBox, B_BYTES = DV / 64 * kBox;
    static constexpr int HALF_BYTES = A_BYTES / 2;                   // of 64 tokens
    static constexpr int SMEM = 1024 + A_BYTES + (TERMS - 1) * HALF_BYTES + B_BYTES;
};

// the largest of a block's values, for every thread
__device__ __forceinline__ float largest(float v, float (&parts)[8])
{
#pragma unroll
    for (int o = 16; o; o /= 2)
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if (threadIdx.x % 32 == 0)
        parts[threadIdx.x / 32] = v;
    __syncthreads();
    for (int i = 0; i < 8; ++i)
        v = fmaxf(v, parts[i]);
    return v;
}

// U = sum_t w_t a_t b_t' of one chunk and head, w_t in [0, 1]: keys and values with w = exp(R_t), or, BACK, queries and gradients of y with
// w = exp(G_t) (there a step of the first token is taken out, so that the largest weight is 1, and put back into the sums).
// One block: rows of 16 bytes are weighted and split where they lie, the further terms beside them for 64 tokens at a time, so that two blocks fit
// into an SM.
template <typename T, int DK, int DV, bool BACK>
__global__ void __launch_bounds__(kThreads, 2) chunk_state_kernel(const AttnDev p, const Rows a, const Rows b, int vec_a, int vec_b, float factor, const float* given)
{
    using S = StateShape<T, DK, DV>;
    __shared__ Control ctl;
    __shared__ Decays dec;
    __shared__ float s_most[8];
    const long long ci = blockIdx.x;
    const int head = blockIdx.y, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    wait_for_previous();
    const Chunk c = chunk_at(p, ci);
    if (c.len <= 0)
        return;
    char* smem = aligned_smem();
    const uint32_t first = smem_u32(smem), rest = first + S::A_BYTES, values = rest + (S::TERMS - 1) * S::HALF_BYTES;
    load_tile<T, DK>(first, a, c, head / p.share, p.dk, vec_a);
    copies_begun();
    load_tile<T, DV>(values, b, c, head, p.dv, vec_b);
    copies_begun();
    if (warp < 4)
        find_decays<T>(p, c, head, dec);
    const uint32_t tmem = set_up(ctl, DV);
    copies_done<1>();
    const float begin = BACK ? dec.g[0] : 0.f;
#pragma unroll
    for (int phase = 0; phase < 2; ++phase) {
#pragma unroll
        for (int i = phase * kChunk * DK / 16; i < (phase + 1) * kChunk * DK / 16; i += kThreads) {
            const int e = i + threadIdx.x, row = e / (DK / 8), c8 = e % (DK / 8);
            float w;
            if (BACK) {
                float sum = dec.g[row] - begin;
                for (int q = 0; q < row / 32; ++q)
                    sum += dec.block[q];
                w = row < c.len ? ex2(sum) : 0.f;
            } else {
                w = to_end(dec, row);
            }
            uint4* at = reinterpret_cast<uint4*>(smem + tile_at(row, c8));
            uint4 term[S::TERMS];
            const uint4 v = *at;
            const uint32_t* in = &v.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float2 x = unpack16<T>(in[j]);
                x.x *= w, x.y *= w;
#pragma unroll
                for (int n = 0; n < S::TERMS; ++n) {
                    const uint32_t u = pack16<T>(x.x, x.y);
                    (&term[n].x)[j] = u;
                    const float2 f = unpack16<T>(u);
                    x.x -= f.x, x.y -= f.y;
                }
            }
            *at = term[0];
            const int low = (c8 / 8) * (kBox / 2) + row % 64 * 128 + (((c8 % 8) ^ (row & 7)) << 4);
#pragma unroll
            for (int n = 1; n < S::TERMS; ++n)
                *reinterpret_cast<uint4*>(smem + S::A_BYTES + (n - 1) * S::HALF_BYTES + low) = term[n];
        }
        if (phase == 0)
            copies_done<0>();
        to_tensor_cores();
        __syncthreads();
        if (warp == 0) {
            constexpr uint32_t id = instruction(kIsBf16<T>, true, true, 128, DV);
            if (elect_one()) {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    mma(tmem, over_tokens(first, phase * 4 + s), over_tokens(values, phase * 4 + s), id, phase > 0 || s > 0);
#pragma unroll
                    for (int n = 1; n < S::TERMS; ++n)
                        mma(tmem, desc(rest + (n - 1) * S::HALF_BYTES + s * 2048, kBox / 2, 1024, 2), over_tokens(values, phase * 4 + s), id, 1);
                }
                commit(smem_u32(&ctl.bar[phase]));
            }
            __syncwarp();
        }
        products_done(ctl, phase);
    }
    const int quarter = warp % 4, half = warp / 4, r = quarter * 32 + lane;
    float most = 0.f;
    if (quarter * 32 < DK) {
        const float f = BACK ? factor * ex2(begin) : factor;
        float4* out = reinterpret_cast<float4*>(p.added) + (ci * p.heads + head) * (long long)(DK * DV / 4) + r;
#pragma unroll
        for (int c0 = 0; c0 < DV / 2; c0 += 32) {
            float v[32];
            tmem_ld32(tmem + half * (DV / 2) + c0 + ((uint32_t)(quarter * 32) << 16), v);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const float4 u = make_float4(v[i] * f, v[i + 1] * f, v[i + 2] * f, v[i + 3] * f);
                most = fmaxf(most, fmaxf(fmaxf(fabsf(u.x), fabsf(u.y)), fmaxf(fabsf(u.z), fabsf(u.w))));
                out[(half * (DV / 2) + c0 + i) / 4 * DK] = u;
            }
        }
    }
    if (!kIsBf16<T>) {
        most = largest(most, s_most);
        if (threadIdx.x == 0)
            p.most[ci * p.heads + head] = most;
        if (given && c.owner >= 0) {
            const long long n = (long long)p.dk * p.dv, at = c.owner * p.heads + head;
            most = 0.f;
            for (long long i = threadIdx.x; i < n; i += kThreads)
                most = fmaxf(most, fabsf(given[at * n + i]));
            most = largest(most, s_most);
            if (threadIdx.x == 0)
                p.most_given[at] = most;
        }
    }
    if (!BACK && threadIdx.x == 0)
        p.whole[ci * p.heads + head] = over_chunk(dec);
    give_back(tmem, DV);
}

// ---- the states in front of the chunks ------------------------------------------------------------------------------------

// S_{c+1} = exp(G_C) S_c + U_c, or, BACK, from the last chunk to the first.  A thread has 8 neighbouring columns of one row of dk; the
// loads of four chunks are under way together.  float16 images are taken times a power of two that a bound on the states' size gives (largest
// |S| so far, decayed, plus the largest |U|), so that they neither overflow nor vanish; `unit` undoes it.
// SPLIT: images of two numbers of 16 bits.
template <typename T, int DK, int DV, bool BACK, bool SPLIT>
__global__ void __launch_bounds__(kThreads) state_scan_kernel(const AttnDev p, const float* added, char* image, const float* given, float* last,
                                                             const float* most, float* unit)
{
    constexpr int IMAGE = DK * DV * 2 * (SPLIT ? 2 : 1), AHEAD = 4;
    wait_for_previous();
    const long long b = blockIdx.x / p.heads;
    const int head = blockIdx.x % p.heads, e = blockIdx.y * kThreads + threadIdx.x, r = e % DK, c0 = e / DK * 8;
    long long first, n;
    if (p.piece_map) {
        first = p.seq_first[b];
        n = p.seq_first[b + 1] - first;
    } else {
        first = b * p.chunks_per_seq;
        n = p.chunks_per_seq;
    }
    const long long place = (b * p.heads + head) * (long long)p.dk * p.dv;
    const long long own = place + (long long)r * p.dv + c0;
    float S[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        S[j] = 0.f;
    if (given && r < p.dk) {
        if (p.vec_state && c0 < p.dv) {
            *reinterpret_cast<float4*>(S) = *reinterpret_cast<const float4*>(given + own);
            *reinterpret_cast<float4*>(S + 4) = *reinterpret_cast<const float4*>(given + own + 4);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < p.dv)
                    S[j] = given[own + j];
        }
    }
    float bound = !kIsBf16<T> && given && n > 0 ? p.most_given[b * p.heads + head] : 0.f;
    for (long long i0 = 0; i0 < n; i0 += AHEAD) {
        float4 u[AHEAD][2];
        float w[AHEAD], m[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const long long c = BACK ? first + n - 1 - (i0 + i) : first + i0 + i, at = c * p.heads + head;
            const bool ok = i0 + i < n;
            const float4* from = reinterpret_cast<const float4*>(added) + (ok ? at : 0) * (long long)(DK * DV / 4) + (long long)(c0 / 4) * DK + r;
            u[i][0] = load_if(from, ok);
            u[i][1] = load_if(from + DK, ok);
            w[i] = load_if(p.whole + (ok ? at : 0), ok);
            m[i] = kIsBf16<T> ? 0.f : load_if(most + (ok ? at : 0), ok);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (i0 + i >= n)
                break;
            const long long c = BACK ? first + n - 1 - (i0 + i) : first + i0 + i, at = c * p.heads + head;
            float up = 1.f;
            if (!kIsBf16<T>) {                   // 2^(13 - floor(log2(bound))): results below 2^14
                const int x = ((__float_as_uint(bound) >> 23) & 255) - 127;
                const int k = min(max(13 - x, -100), 100);
                up = __uint_as_float((uint32_t)(k + 127) << 23);
                if (blockIdx.y == 0 && threadIdx.x == 0)
                    unit[at] = __uint_as_float((uint32_t)(127 - k) << 23);
                bound = fmaf(w[i], bound, m[i]);
            }
            uint4 hi, lo;
            uint32_t *h = &hi.x, *l = &lo.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = S[2 * j] * up, y = S[2 * j + 1] * up;
                h[j] = pack16<T>(x, y);
                if (SPLIT) {
                    const float2 f = unpack16<T>(h[j]);
                    l[j] = pack16<T>(x - f.x, y - f.y);
                }
            }
            char* to = image + at * IMAGE + ((c0 / 8) * DK + r) * 16;
            *reinterpret_cast<uint4*>(to) = hi;
            if (SPLIT)
                *reinterpret_cast<uint4*>(to + DK * DV * 2) = lo;
            const float* f = &u[i][0].x;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                S[j] = fmaf(w[i], S[j], f[j]);
        }
    }
    if (last && r < p.dk) {
        if (p.vec_state && c0 < p.dv) {
            *reinterpret_cast<float4*>(last + own) = *reinterpret_cast<const float4*>(S);
            *reinterpret_cast<float4*>(last + own + 4) = *reinterpret_cast<const float4*>(S + 4);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < p.dv)
                    last[own + j] = S[j];
        }
    }
}

// ---- outputs --------------------------------------------------------------------------------------------------------------

// Decay of the pairs (row, 32 columns of block b) of the lower triangle times f: a row's lane has `mine` = its sum from its block's begin.
// `to_here` [32]: exp from each column to the begin of the row's block.
__device__ __forceinline__ void decay_row(float (&v)[32], const Decays& d, bool diagonal, int b, int lane, float mine, float e_mine, const float* to_here)
{
    if (diagonal) {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const float4 g = *reinterpret_cast<const float4*>(d.g + b * 32 + j);
            v[j] = j <= lane ? v[j] * ex2(mine - g.x) : 0.f;
            v[j + 1] = j + 1 <= lane ? v[j + 1] * ex2(mine - g.y) : 0.f;
            v[j + 2] = j + 2 <= lane ? v[j + 2] * ex2(mine - g.z) : 0.f;
            v[j + 3] = j + 3 <= lane ? v[j + 3] * ex2(mine - g.w) : 0.f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const float4 t = *reinterpret_cast<const float4*>(to_here + j);
            v[j] *= e_mine * t.x;
            v[j + 1] *= e_mine * t.y;
            v[j + 2] *= e_mine * t.z;
            v[j + 3] *= e_mine * t.w;
        }
    }
}

template <int DK, int DV> struct OutShape {
    static constexpr int Q_BYTES = DK / 64 * kBox, V_BYTES = DV / 64 * kBox, KV_BYTES = Q_BYTES > V_BYTES ? Q_BYTES : V_BYTES;
    static constexpr int QY_BYTES = KV_BYTES;    // queries, then the staged results
    static constexpr int IMAGE = DK * DV * 2;
    static constexpr int SMEM = 1024 + QY_BYTES + KV_BYTES + IMAGE;
};

__device__ __forceinline__ void load_image(uint32_t to, const char* from, int bytes)
{
    for (int i = threadIdx.x * 16; i < bytes; i += kThreads * 16)
        copy16(to + i, from + i, true);
}

// One chunk of one head: scores and q S_0 into tensor memory; the scores, times their decays, go back there in 16 bits as an operand, and
// the values take the keys' place in shared memory meanwhile.  Two blocks to an SM, so that one's loads run beside the other's products.
template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads, 2) chunk_out_kernel(const AttnDev p)
{
    using S = OutShape<DK, DV>;
    __shared__ Control ctl;
    __shared__ Decays dec;
    __shared__ alignas(16) float s_to[4][96];                // [block][earlier token]: decay from it to the block's begin
    const long long ci = blockIdx.x;
    const int head = blockIdx.y, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, quarter = warp % 4, half = warp / 4;
    wait_for_previous();
    const Chunk c = chunk_at(p, ci);
    if (c.len <= 0)
        return;
    char* smem = aligned_smem();
    const uint32_t queries = smem_u32(smem), keys = queries + S::QY_BYTES, image = keys + S::KV_BYTES;
    load_tile<T, DK>(queries, p.q, c, head / p.share, p.dk, p.vec_q);
    load_tile<T, DK>(keys, p.k, c, head / p.share, p.dk, p.vec_k);
    load_image(image, p.image + (ci * p.heads + head) * (long long)S::IMAGE, S::IMAGE);
    copies_begun();
    if (warp < 4)
        find_decays<T>(p, c, head, dec);
    const uint32_t tmem = set_up(ctl, 256);      // scores: columns 0 .. 127, results behind them
    const uint32_t scores = tmem, results = tmem + 128, lanes = (uint32_t)(quarter * 32) << 16;
    for (int i = threadIdx.x; i < 4 * 96; i += kThreads)
        s_to[i / 96][i % 96] = i % 96 < i / 96 * 32 ? to_block(dec, i % 96, i / 96) : 0.f;
    copies_done<0>();
    to_tensor_cores();
    __syncthreads();
    if (warp == 0) {
        constexpr uint32_t id_scores = instruction(kIsBf16<T>, false, false, 128, 128), id_state = instruction(kIsBf16<T>, false, true, 128, DV);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < DK / 16; ++s)
                mma(scores, over_columns(queries, s), over_columns(keys, s), id_scores, s > 0);
            commit(smem_u32(&ctl.bar[0]));
#pragma unroll
            for (int s = 0; s < DK / 16; ++s)
                mma(results, over_columns(queries, s), image_over_dk<DK>(image, s), id_state, s > 0);
            commit(smem_u32(&ctl.bar[1]));
        }
        __syncwarp();
    }
    products_done(ctl, 0);
    load_tile<T, DV>(keys, p.v, c, head, p.dv, p.vec_v);
    copies_begun();
    const int row = quarter * 32 + lane;
    const float mine = dec.g[row], e_mine = ex2(mine);
    uint32_t packed[2][16];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int b = half + 2 * i;
        if (b <= quarter) {
            float v[32];
            tmem_ld32(scores + b * 32 + lanes, v);
            decay_row(v, dec, b == quarter, b, lane, mine, e_mine, &s_to[quarter][b < quarter ? b * 32 : 0]);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                packed[i][j] = pack16<T>(v[2 * j] * p.scale, v[2 * j + 1] * p.scale);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                packed[i][j] = 0;
        }
    }
    // both warps of these rows have read what is overwritten now
    before_barrier();
    asm volatile("bar.sync %0, 64;" :: "r"(1 + quarter) : "memory");
    behind_barrier();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        tmem_st16(scores + (half + 2 * i) * 16 + lanes, packed[i]);
    products_done(ctl, 1);
    {
        const float f = from_begin(dec, row) * p.scale * (kIsBf16<T> ? 1.f : p.unit[ci * p.heads + head]);
#pragma unroll
        for (int c0 = 0; c0 < DV / 2; c0 += 32) {
            float v[32];
            const uint32_t at = results + half * (DV / 2) + c0 + lanes;
            tmem_ld32(at, v);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                v[j] *= f;
            tmem_st32(at, v);
        }
    }
    tmem_st_done();
    copies_done<0>();
    to_tensor_cores();
    before_barrier();
    __syncthreads();
    if (warp == 0) {
        behind_barrier();
        constexpr uint32_t id = instruction(kIsBf16<T>, false, true, 128, DV);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < 8; ++s)
                mma_tmem(results, scores + s * 8, over_tokens(keys, s), id, 1);
            commit(smem_u32(&ctl.bar[2]));
        }
        __syncwarp();
    }
    products_done(ctl, 2);
#pragma unroll
    for (int c0 = 0; c0 < DV / 2; c0 += 32) {
        float v[32];
        tmem_ld32(results + half * (DV / 2) + c0 + lanes, v);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
            const uint4 w = make_uint4(pack16<T>(v[j], v[j + 1]), pack16<T>(v[j + 2], v[j + 3]), pack16<T>(v[j + 4], v[j + 5]), pack16<T>(v[j + 6], v[j + 7]));
            *reinterpret_cast<uint4*>(smem + tile_at(row, (half * (DV / 2) + c0 + j) / 8)) = w;
        }
    }
    give_back(tmem, 256);
    store_tile<T, DV>(smem, p.y, c, head, p.dv, p.vec_y);
}

// ---- one token of each sequence -------------------------------------------------------------------------------------------

constexpr int kStepThreads = 128;

// The state is read and written once, which is all that counts.  A block has all rows and COLS columns of a head's state: a thread 4 columns
// (V = 4; 1 where states cannot be accessed by 16 bytes) of every PARTS-th row, in loads of eight rows that are under way together.
template <typename T, int V>
__global__ void __launch_bounds__(kStepThreads) decay_step_kernel(const AttnDev p, int lanes)
{
    __shared__ float s_q[128], s_k[128];
    __shared__ float s_y[kStepThreads * V];
    wait_for_previous();
    const long long b = blockIdx.x / p.heads;
    const int head = blockIdx.x % p.heads, group = head / p.share;
    const int sub = threadIdx.x % lanes, part = threadIdx.x / lanes, parts = kStepThreads / lanes;
    const int c0 = (blockIdx.y * lanes + sub) * V;
    const bool have = c0 < p.dv;
    for (int i = threadIdx.x; i < p.dk; i += kStepThreads) {
        s_q[i] = to_f(row_ptr<T>(p.q, b, 0)[(long long)group * p.dk + i]) * p.scale;
        s_k[i] = to_f(row_ptr<T>(p.k, b, 0)[(long long)group * p.dk + i]);
    }
    const float d = p.delta.ptr ? step_of(p, raw_step<T>(p, b, 0, head)) : 1.f;
    const float a = ex2(p.A[head] * d * kLog2e + kExBias);
    float v[V], y[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        v[j] = have ? to_f(row_ptr<T>(p.v, b, 0)[(long long)head * p.dv + c0 + j]) : 0.f;
        y[j] = 0.f;
    }
    float* S = p.state_out + (b * p.heads + head) * (long long)p.dk * p.dv + c0;
    __syncthreads();
    for (int r0 = part; r0 < p.dk; r0 += 8 * parts) {
        Vec<float, V> h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            h[i] = load_if(reinterpret_cast<const Vec<float, V>*>(S + (long long)(r0 + i * parts) * p.dv), have && r0 + i * parts < p.dk);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + i * parts;
            if (have && r < p.dk) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[i].v[j] = fmaf(a, h[i].v[j], s_k[r] * v[j]);
                    y[j] = fmaf(s_q[r], h[i].v[j], y[j]);
                }
                *reinterpret_cast<Vec<float, V>*>(S + (long long)r * p.dv) = h[i];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
        s_y[part * lanes * V + sub * V + j] = y[j];
    __syncthreads();
    for (int i = threadIdx.x; i < lanes * V; i += kStepThreads) {
        const int c = blockIdx.y * lanes * V + i;
        if (c < p.dv) {
            float sum = 0.f;
            for (int q = 0; q < parts; ++q)
                sum += s_y[q * lanes * V + i];
            row_ptr<T>(p.y, b, 0)[(long long)head * p.dv + c] = from_f<T>(sum);
        }
    }
}

} // namespace dattn
} // namespace ttc
