// Linear attention with a decay for each head:  S_t = exp(l_t) S_{t-1} + k_t v_t',  y_t = scale q_t S_t,  l_t = A D_t.
//
// Token by token this is 5 dk dv operations on a state that no register file holds.  Over a chunk of 128 tokens, with
// G_i = l_1 + .. + l_i from the chunk's first token and R_j = l_{j+1} + .. + l_128, it is
//
//     y_i = scale [ sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j  +  exp(G_i) q_i S_0 ],      S_C = exp(G_C) S_0 + sum_j exp(R_j) k_j v_j'
//
// four products of 128 rows each, which the 5th-generation tensor cores take, and the chunks depend on one another through S only:
//
//     walk_kernel          y, chunk by chunk along a sequence (or a piece of one), S in registers
//     state_walk_kernel    S alone: what a piece adds to it, where sequences are cut into pieces; for the gradients, S in front of every chunk
//     join_kernel          S in front of the pieces, from what each adds
//     decay_step_kernel    one token: token by token after all
//
// Exponents.  None is positive: pairs of tokens of one block of 32 take exp(G_i - G_j) itself, from sums within the block; others the product
// of exp(from the block's begin to i) and exp(from j to that begin), so that no difference of long sums is formed.  Exponents
// below -192 / log2(e) count as that (their exponentials are zero), so that a decay of minus infinity, which forgets
// everything, gives no difference of infinities.  The sums within a block reach 32 times that, where float32's steps are 5e-4: what their additions round off is
// carried along in a second number, so that a difference of two of them is off by its own rounding alone, whatever stands in front of both tokens (with one number 25 tokens that
// forget, in front of seven that do not, put dA off by 1.2e-5 of the sum of its terms' magnitudes).
//
// Roundings.  Sums are float32 in tensor memory, states float32.  Operands of the tensor cores are 16 bits: scores with their decay, and S_0 where q
// multiplies it, are rounded once (half a step each, as the result itself; float16: times a power of two, of a row of scores or of the state, so that neither small nor large ones
// lose more: 16381 tokens of 8 heads of 64 x 64 took 63.6 us without the rows', 66.5 with them).  The weighted values of S_C are not: states are float32 results and are carried on, so
// the values go in as a sum of numbers of 16 bits, each what the ones before it left: three bfloat16 or two float16 (2^-24, 2^-22 of the value; two bfloat16 leave 2^-18,
// and the states were off by 2.4e-6 in the 2-norm).
#pragma once

#include <cuda.h>

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
    const int2* piece_map;                       // packed sequences, gradients: sequence and first token of each chunk
    const int* seq_first;                        // and the first chunk of each sequence
    long long chunks_per_seq, chunks;            // equal sequences; chunks in all (packed: room for them)
    long long piece, pieces_per_seq, pieces;     // tokens of a piece; the same for pieces
    int heads, share, dk, dv;                    // share: heads of a group
    int softplus;
    float scale;
    Rows q, k, v, delta, y;
    int head_q, head_k, head_v;                  // elements from a head to the next one: its channels, or those rounded up, of rows laid out anew
    int vec_y;                                   // bytes that results can be accessed by: 16, 8 or 2
    int vec_state;                               // states can be accessed by 16 bytes
    const float *A, *delta_bias, *state;
    float* state_out;
    const float* piece_state;                    // scratch: the states in front of the pieces of a sequence
};

struct Chunk {
    long long seq, row0;                         // sequence and row of the first token, as row_ptr takes them
    int len;                                     // tokens, 0: nothing to do
};

__device__ __forceinline__ Chunk chunk_at(const AttnDev& p, long long c)
{
    Chunk r;
    if (p.piece_map) {
        const int2 m = p.piece_map[c];
        if (m.x < 0)
            return Chunk{0, 0, 0};
        const Span s = span_of(p.seqs, m.x);
        r.seq = 0;
        r.row0 = s.row0 + m.y;
        r.len = (int)min(s.len - m.y, (long long)kChunk);
    } else {
        r.seq = c / p.chunks_per_seq;
        r.row0 = (c % p.chunks_per_seq) * kChunk;
        r.len = (int)min(p.seqs.tokens - r.row0, (long long)kChunk);
    }
    return r;
}

// ---- decays of a chunk --------------------------------------------------------------------------------------------------

struct alignas(16) Decays {
    float g[kChunk];                             // sums to the base 2 from the begin of the token's block of 32, the token's own included
    float low[kChunk];                           // what their additions rounded off
    float s[kChunk];                             // behind the token, to the end of its block
    float block[4];                              // of whole blocks
};

__device__ __forceinline__ float step_of(const AttnDev& p, float raw) { return p.softplus ? softplus(raw) : raw; }

// What softplus or nothing is taken of, and the step; raw only where there is a delta.
template <typename T> __device__ __forceinline__ float raw_step(const AttnDev& p, long long seq, long long row, int head)
{
    return to_f(row_ptr<T>(p.delta, seq, row)[head]) + (p.delta_bias ? p.delta_bias[head] : 0.f);
}

// A of a head.  Minus infinity becomes the lowest number: times a step of 0 (a softplus that underflows) it has to be 0.
__device__ __forceinline__ float rate(const AttnDev& p, int head) { return p.A[head] < -3.4e38f ? -3.4e38f : p.A[head]; }
__device__ __forceinline__ float log_decay(float A, float step)
{
    const float l = A * step * kLog2e;
    return l < kFloor ? kFloor : l;              // NaN stays
}
template <typename T> __device__ __forceinline__ float log_decay_at(const AttnDev& p, const Chunk& c, int head, int t)
{
    return t < c.len ? log_decay(rate(p, head), p.delta.ptr ? step_of(p, raw_step<T>(p, c.seq, c.row0 + t, head)) : 1.f) : 0.f;
}

// By one warp for the 32 tokens of a block, from the log decay of each lane's token: the sum from the block's begin, and behind the token to its end.  LOW: what the additions of the
// first one rounded off, too (by Knuth's sum of two numbers with its rounding error).
template <bool LOW> __device__ __forceinline__ float block_sums(float l, float& behind, float& low)
{
    const int lane = threadIdx.x % 32;
    float g = l, s = l;
    low = 0.f;
#pragma unroll
    for (int i = 1; i < 32; i *= 2) {
        const float up = __shfl_up_sync(0xffffffffu, g, i), b = __shfl_down_sync(0xffffffffu, s, i);
        const float a = lane >= i ? up : 0.f, sum = g + a;
        if (LOW) {
            const float up_low = __shfl_up_sync(0xffffffffu, low, i), part = sum - g;
            low += (lane >= i ? up_low : 0.f) + ((g - (sum - part)) + (a - part));
        }
        g = sum;
        s += lane + i < 32 ? b : 0.f;
    }
    s = __shfl_down_sync(0xffffffffu, s, 1);
    behind = lane < 31 ? s : 0.f;
    return g;
}
__device__ __forceinline__ void block_decays(float l, int t, Decays& o)
{
    o.g[t] = block_sums<true>(l, o.s[t], o.low[t]);
    if (t % 32 == 31)
        o.block[t / 32] = o.g[t];
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

// `width` channels from channel col0 of the rows, for the last chunk of a packed sequence, which others' rows follow: the copy engine fills the others.  (Channels behind a head's up to
// eight are zeros, as align_kernel lays them out.)
template <typename T, int COLS, int THREADS>
__device__ __forceinline__ void load_tile(uint32_t to, const Rows& r, const Chunk& c, int col0, int width, int thread)
{
    const T* base = row_ptr<T>(r, c.seq, c.row0) + col0;
#pragma unroll 8
    for (int i = 0; i < kChunk * COLS / 8; i += THREADS) {
        const int e = i + thread, row = e / (COLS / 8), c8 = e % (COLS / 8);
        const bool ok = row < c.len && c8 * 8 < width;
        copy16(to + tile_at(row, c8), ok ? base + row * r.ts + c8 * 8 : base, ok);
    }
}

// The tile of results staged in shared memory, to its rows.
template <typename T, int COLS, int THREADS> __device__ __forceinline__ void store_tile(const char* from, const Rows& r, const Chunk& c, int head, int width, int vec)
{
    T* base = row_ptr<T>(r, c.seq, c.row0) + (long long)head * width;
    constexpr int N = kChunk * COLS / 8 / THREADS;                   // vectors of a thread: of one place in every THREADS / (COLS / 8)-th row
    const int c8 = threadIdx.x % (COLS / 8), row0 = threadIdx.x / (COLS / 8);
    if (c8 * 8 >= width)
        return;
    uint4 w[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        w[i] = *reinterpret_cast<const uint4*>(from + tile_at(row0 + i * (THREADS / (COLS / 8)), c8));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = row0 + i * (THREADS / (COLS / 8));
        T* at = base + row * r.ts + c8 * 8;
        if (row >= c.len)
            break;
        if (vec == 16) {
            *reinterpret_cast<uint4*>(at) = w[i];
        } else if (vec == 8) {
            *reinterpret_cast<uint2*>(at) = make_uint2(w[i].x, w[i].y);
            if (c8 * 8 + 4 < width)
                *reinterpret_cast<uint2*>(at + 4) = make_uint2(w[i].z, w[i].w);
        } else {
            const Vec<T, 8> u = *reinterpret_cast<const Vec<T, 8>*>(&w[i]);
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
// N products of 16 indices each, one behind the other; STEP: 16 bytes from an operand's 16 indices to the next ones.  Rolled up, as whatever need not lie in registers here: a block goes
// through its code once, and waited for instructions more than for anything else (the tensor cores take 64 clocks for one of these).
constexpr int kColumns = 0, kTokens = 128;                           // (over columns: 2, and from box to box)
template <int STEP> __device__ __forceinline__ uint64_t step_to(int s) { return STEP == kColumns ? (s / 4) * (kBox >> 4) + (s % 4) * 2 : s * STEP; }
template <int N, int A, int B> __device__ __forceinline__ void products(uint32_t d, uint64_t a, uint64_t b, uint32_t id, bool add)
{
#pragma unroll 1
    for (int s = 0; s < N; ++s)
        mma(d, a + step_to<A>(s), b + step_to<B>(s), id, add || s > 0);
}
template <int N, int B> __device__ __forceinline__ void products_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t id)
{
#pragma unroll 1
    for (int s = 0; s < N; ++s)
        mma_tmem(d, a + s * 8, b + step_to<B>(s), id, 1);
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, float (&v)[16])
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i)
        v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld8(uint32_t at, float (&v)[8])
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st4(uint32_t at, const uint32_t (&r)[4])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                    "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
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

// In pairs: half the instructions of a loop over the numbers.
template <int N> __device__ __forceinline__ void scale_all(float (&v)[N], float f)
{
#pragma unroll
    for (int j = 0; j < N; j += 2)
        unpack2(mul2(pack2(v[j], v[j + 1]), pack2(f, f)), v[j], v[j + 1]);
}
template <int N> __device__ __forceinline__ void add_all(float (&v)[N], const float (&w)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 2)
        unpack2(add2(pack2(v[j], v[j + 1]), pack2(w[j], w[j + 1])), v[j], v[j + 1]);
}
// S = over S + u
template <int N> __device__ __forceinline__ void carry_all(float (&S)[N], float over, const float (&u)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 2)
        unpack2(fma2(pack2(over, over), pack2(S[j], S[j + 1]), pack2(u[j], u[j + 1])), S[j], S[j + 1]);
}

template <typename T> constexpr bool kIsBf16 = std::is_same<T, bf16>::value;

// A pair of numbers times w as a sum of TERMS pairs of 16 bits, each what those before it left.  bfloat16 cuts off instead of rounding: three times 8 bits are
// all of the product's 24, and take no conversions.
template <typename T, int TERMS, typename F> __device__ __forceinline__ void split_terms(uint32_t pair, float w, F&& put)
{
    const float2 in = unpack16<T>(pair);
    f2 x = mul2(pack2(in.x, in.y), pack2(w, w));
#pragma unroll
    for (int n = 0; n < TERMS; ++n) {
        float a, b;
        unpack2(x, a, b);
        float2 f;
        if (kIsBf16<T>) {
            put(n, __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632));
            f = make_float2(__uint_as_float(__float_as_uint(a) & 0xffff0000u), __uint_as_float(__float_as_uint(b) & 0xffff0000u));
        } else {
            const uint32_t u = pack16<T>(a, b);
            put(n, u);
            f = unpack16<T>(u);
        }
        if (n + 1 < TERMS)
            x = fma2(pack2(f.x, f.y), pack2(-1.f, -1.f), x);
    }
}

extern __shared__ __align__(1024) char dattn_tiles[];

// Barriers and tensor memory of a block.
struct Control {
    uint64_t bar[3];
    uint32_t tmem;
    int dead;
};

// Behind wait_for_previous, as in every kernel here: blocks that held tensor memory while they wait would keep it from those of the kernel in front on the same SM.
__device__ __forceinline__ uint32_t set_up(Control& c, int columns)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < 3; ++i)
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
// Decay of the pairs of a row and 32 tokens of another block, in a row's lane: e_row, the row's decay to that block, times each token's decay within it.
__device__ __forceinline__ void decay_earlier(float (&v)[32], float e_row, const float* within)
{
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        const float4 t = *reinterpret_cast<const float4*>(within + j);
        unpack2(mul2(pack2(v[j], v[j + 1]), mul2(pack2(e_row, e_row), pack2(t.x, t.y))), v[j], v[j + 1]);
        unpack2(mul2(pack2(v[j + 2], v[j + 3]), mul2(pack2(e_row, e_row), pack2(t.z, t.w))), v[j + 2], v[j + 3]);
    }
}
// ---- rows laid out anew ---------------------------------------------------------------------------------------------------

// Operands that the copy engines cannot take (heads that do not begin on 16 bytes, one row for all tokens) are copied first, the heads' channels rounded up to eight with zeros behind them.
// 64 threads that read a chunk's tiles by elements were the other way: 4 x 1024 tokens of 16 heads of 36 x 36 took 263 us, now 42, of 37 x 37 259 and 56, of 100 x 100 421 and 60; 3 x 29 tokens
// of 6 heads of 36 x 20 13.7 and 10.6.
struct Operands {
    struct {
        Rows from;
        unsigned short* to;
        int heads, width, padded, vec;           // vec: bytes that rows can be read by: 8 or 2
    } of[4];
    int n;
};
constexpr int kAlignRows = 8;                    // of a block
static __global__ void __launch_bounds__(256) align_kernel(const Seqs s, const Operands o)
{
    wait_for_previous();
    const auto& q = o.of[blockIdx.y];
    const unsigned each = q.padded / 8, per_row = q.heads * each;
    const long long rows = s.offsets ? s.tokens : s.batch * s.tokens;
    for (long long row0 = (long long)blockIdx.x * kAlignRows; row0 < rows; row0 += (long long)gridDim.x * kAlignRows) {
        uint4* to = reinterpret_cast<uint4*>(q.to + row0 * q.heads * q.padded);
        const unsigned n = per_row * (unsigned)min((long long)kAlignRows, rows - row0);
        for (unsigned e = threadIdx.x; e < n; e += 256) {
            const long long row = row0 + e / per_row, seq = s.offsets ? 0 : row / s.tokens;
            const unsigned head = e % per_row / each, c = e % each * 8;
            const unsigned short* from = row_ptr<unsigned short>(q.from, seq, row - seq * s.tokens) + (long long)head * q.width + c;
            if (q.vec == 8) {
                const uint2 a = *reinterpret_cast<const uint2*>(from), b = load_if(reinterpret_cast<const uint2*>(from + 4), c + 4 < q.width);
                to[e] = make_uint4(a.x, a.y, b.x, b.y);
            } else {
                Vec<unsigned short, 8> u;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    u.v[j] = load_if(from + j, c + j < q.width);
                to[e] = *reinterpret_cast<const uint4*>(&u);
            }
        }
    }
}

// ---- a walk along the chunks ----------------------------------------------------------------------------------------------

constexpr int kWalkThreads = 512;
constexpr int kCols = 64;                        // value channels of a walk: heads of more are walked along twice

// A piece of a sequence (all of it, where there are enough sequences and heads), and the state in registers: of kWalkThreads threads, each has 16 neighbouring columns of
// a row of dk.
struct Piece {
    long long seq, row0;                         // as a Chunk's
    long long owner;                             // the sequence
    long long t0, len;                           // its first token in the sequence, and its tokens
    bool first, last;                            // of its sequence
};

// What a block of a walk works for: pieces one after the other, the heads and columns of each together.
struct Place {
    long long piece;
    int head, part;                              // part of `parts`: columns, or the way
};
__device__ __forceinline__ Place place_of(const AttnDev& p, int parts)
{
    const unsigned id = blockIdx.x, each = p.heads * parts;
    return Place{id / each, (int)(id % each / parts), (int)(id % parts)};
}

// Piece i, found by a whole warp: of packed sequences, which have one piece at least, by going along their lengths 32 at a time.  (`first_of_sequence`: number of its sequence's
// first piece.)  Offsets that decrease leave lengths of nothing.
__device__ __forceinline__ Piece piece_at(const AttnDev& p, long long i, long long* first_of_sequence = nullptr)
{
    Piece r = {0, 0, -1, 0, 0, false, false};
    if (p.seqs.offsets) {
        const int lane = threadIdx.x % 32;
        if (p.pieces == p.seqs.batch && p.seqs.batch > 32) {         // uncut (going along the lengths, 16384 sequences of 4 tokens took 109 ms, now 6.5)
            const Span s = span_of(p.seqs, i);
            r.owner = i;
            r.row0 = s.row0;
            r.len = s.len;
            r.first = r.last = true;
            return r;
        }
        if (p.pieces == p.seqs.batch) {
            // the longest first, so that no long one is left for the end (7 sequences of 4093 tokens in all, 32 walks each: 60 -> 47 us)
            const Span s = lane < p.seqs.batch ? span_of(p.seqs, lane) : Span{0, -1};
            int rank = 0;
#pragma unroll
            for (int o = 0; o < 32; ++o) {
                const long long v = __shfl_sync(0xffffffffu, s.len, o);
                rank += v > s.len || (v == s.len && o < lane);
            }
            const int at = __ffs(__ballot_sync(0xffffffffu, rank == i)) - 1;
            r.owner = at;
            r.row0 = __shfl_sync(0xffffffffu, s.row0, at);
            r.len = __shfl_sync(0xffffffffu, s.len, at);
            r.first = r.last = true;
            return r;
        }
        long long base = 0;
        for (long long b0 = 0; b0 < p.seqs.batch; b0 += 32) {
            const long long b = b0 + lane;
            const Span s = b < p.seqs.batch ? span_of(p.seqs, b) : Span{0, 0};
            const int own = b < p.seqs.batch ? (int)max((s.len + p.piece - 1) / p.piece, 1ll) : 0;
            int sum = own;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                sum += lane >= o ? v : 0;
            }
            const unsigned here = __ballot_sync(0xffffffffu, i < base + sum);
            if (here) {
                const int at = __ffs(here) - 1;
                const long long row0 = __shfl_sync(0xffffffffu, s.row0, at), len = __shfl_sync(0xffffffffu, s.len, at);
                const long long first = base + __shfl_sync(0xffffffffu, sum - own, at), t0 = (i - first) * p.piece;
                if (first_of_sequence)
                    *first_of_sequence = first;
                r.owner = b0 + at;
                r.row0 = row0 + t0;
                r.t0 = t0;
                r.len = min(len - t0, p.piece);
                r.first = t0 == 0;
                r.last = t0 + p.piece >= len;
                return r;
            }
            base += __shfl_sync(0xffffffffu, sum, 31);
        }
    } else {
        r.seq = r.owner = i / p.pieces_per_seq;
        r.row0 = r.t0 = i % p.pieces_per_seq * p.piece;
        r.len = min(p.seqs.tokens - r.row0, p.piece);
        r.first = r.row0 == 0;
        r.last = r.row0 + p.piece >= p.seqs.tokens;
    }
    return r;
}
__device__ __forceinline__ Chunk chunk_of(const Piece& q, int i)
{
    return Chunk{q.seq, q.row0 + (long long)i * kChunk, (int)min(q.len - (long long)i * kChunk, (long long)kChunk)};
}

// The columns of a row of a float32 state that a thread has, from or to [batch][heads][dk][dv].
template <int N> __device__ __forceinline__ void load_state(float (&S)[N], const AttnDev& p, const float* from, long long owner, int head, int row, int c0)
{
#pragma unroll
    for (int j = 0; j < N; ++j)
        S[j] = 0.f;
    if (!from || row >= p.dk)
        return;
    from += ((owner * p.heads + head) * p.dk + row) * (long long)p.dv;
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        if (p.vec_state && c0 + j < p.dv) {
            *reinterpret_cast<float4*>(S + j) = *reinterpret_cast<const float4*>(from + c0 + j);
        } else {
#pragma unroll
            for (int i = j; i < j + 4; ++i)
                if (c0 + i < p.dv)
                    S[i] = from[c0 + i];
        }
    }
}
template <int N> __device__ __forceinline__ void store_state(const float (&S)[N], const AttnDev& p, float* to, long long owner, int head, int row, int c0)
{
    if (!to || row >= p.dk)
        return;
    to += ((owner * p.heads + head) * p.dk + row) * (long long)p.dv;
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        if (p.vec_state && c0 + j < p.dv) {
            *reinterpret_cast<float4*>(to + c0 + j) = *reinterpret_cast<const float4*>(S + j);
        } else {
#pragma unroll
            for (int i = j; i < j + 4; ++i)
                if (c0 + i < p.dv)
                    to[c0 + i] = S[i];
        }
    }
}

constexpr int kFrontWarps = 2;                   // that load, and find the decays of two blocks of 32 tokens each (with a third, threads would have 80 registers)
constexpr int kWalkBlock = kWalkThreads + 32 * (kFrontWarps + 1);
constexpr int kWalkWarps = kWalkThreads / 32;

// What a walk needs of a chunk's decays: exponentials within blocks of 32 tokens and over whole blocks, to be multiplied.
struct alignas(16) Table {
    float g[kChunk];                             // sums to the base 2 from the begin of the token's block, the token's own included
    float to_end[kChunk];                        // exp from behind the token to its block's end
    float block[4];                              // sums over the blocks
    float before[4], behind[4];                  // exp over all blocks before and behind one
    float skipped[4];                            // over blocks 1, 1 and 2, 2: between two that are not neighbours (index a + b - 2)
    float whole;
};
__device__ __forceinline__ float between(const Table& t, int a, int b) { return b - a < 2 ? 1.f : t.skipped[a + b - 2]; }

template <typename T, int DK> struct WalkShape {
    static constexpr int TERMS = kIsBf16<T> ? 3 : 2;                 // numbers of 16 bits that a weighted value is split into
    static constexpr int K_BYTES = DK / 64 * kBox, V_BYTES = kBox, STAGE = 2 * K_BYTES + V_BYTES;
    static constexpr int IMAGE = DK * kCols * 2;
    struct Small {
        uint64_t loaded[2], freed[2];            // of the two stages
        uint64_t scores, state, added, out;      // products that are done
        uint64_t weighted, weighed, imaged;      // operands that are there: weighted values, weighted scores (and q S_0 times its decays), the image of the state
        uint64_t drained;
        uint32_t tmem;
        int dead;
        Table dec[2];
        alignas(8) float low[2][kIsBf16<T> ? 2 : kChunk];            // of the sums within blocks: what their additions rounded off (up to 2e-4, of weights that bfloat16 rounds by 2e-3)
        float most[kIsBf16<T> ? 1 : 32], row_most[4][kIsBf16<T> ? 1 : kChunk];
    };
    static constexpr int TILES = 2 * STAGE + TERMS * V_BYTES + IMAGE;
    static constexpr int SMEM = TILES + sizeof(Small);
    static constexpr int COLUMNS = 512;                              // of tensor memory
};
static_assert(WalkShape<bf16, 128>::SMEM <= 232448 && WalkShape<__half, 128>::SMEM <= 232448, "shared memory of a block");

// a power of two that takes `most` to 2^13 .. 2^14, and its inverse
__device__ __forceinline__ float power_for(float most, float& inverse)
{
    const int x = (int)((__float_as_uint(most) >> 23) & 255) - 127, k = min(max(13 - x, -100), 100);
    inverse = __uint_as_float((uint32_t)(127 - k) << 23);
    return __uint_as_float((uint32_t)(127 + k) << 23);
}
// the largest of the walking threads' values; `parts` may be written again behind the threads' next barrier
__device__ __forceinline__ float walk_largest(float v, float* parts)
{
#pragma unroll
    for (int o = 16; o; o /= 2)
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (threadIdx.x % 32 == 0)
        parts[threadIdx.x / 32] = v;
    asm volatile("bar.sync 1, %0;" :: "n"(kWalkThreads) : "memory");
    for (int i = 0; i < kWalkWarps; ++i)
        v = fmaxf(v, parts[i]);
    return v;
}

// float16: weights of a row (scores times decays) go into their product times a power of two, the row's, so that they neither overflow nor vanish: `most`, the largest
// of them, is taken to 2^13 .. 2^14, or towards there by `highest` at most.  A product of the smallest numbers, 2^-48, is held to 11 bits that way.
constexpr int kHighest = 60;
__device__ __forceinline__ float row_power(float most, int highest, float& inverse)
{
    const int x = (int)((__float_as_uint(most) >> 23) & 255) - 127, k = min(max(13 - x, -100), highest);
    inverse = __uint_as_float((uint32_t)(127 - k) << 23);
    return __uint_as_float((uint32_t)(127 + k) << 23);
}
// (times the state's power of two, `unit`, it stays below 2^60, so that what the state gives to the row, and its product with another in the gradients, stays in float32)
__device__ __forceinline__ int highest_with(float unit) { return min(kHighest, kHighest - ((int)(__float_as_uint(unit) >> 23) - 127)); }
template <int N> __device__ __forceinline__ float largest(const float (&v)[N])
{
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j)
        m = fmaxf(m, fabsf(v[j]));
    return m;
}
// Weights as 16-bit numbers.  float16: times a power of two of their own, of which `inverse` is left, until the row's is known (`change`: that one over theirs, 1 at most).
template <typename T, int N> __device__ __forceinline__ void pack_weights(const float (&v)[N], uint32_t (&to)[N / 2], float& most, float& inverse)
{
    float up = 1.f;
    if (!kIsBf16<T>) {
        most = largest(v);
        up = row_power(most, kHighest, inverse);
    }
#pragma unroll
    for (int j = 0; j < N / 2; ++j)
        to[j] = kIsBf16<T> ? pack16<T>(v[2 * j], v[2 * j + 1]) : pack16<T>(v[2 * j] * up, v[2 * j + 1] * up);
}
template <int N> __device__ __forceinline__ void change_power(uint32_t (&v)[N], float change)
{
    const __half2 f = __float2half2_rn(change);  // (2^-24 at least, or nothing)
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&v[j]), f);
        v[j] = *reinterpret_cast<const uint32_t*>(&r);
    }
}

// Rows as [batch][tokens][heads][channels] for the copy engines.
struct Maps {
    CUtensorMap q, k, v;
};
__device__ __forceinline__ void fetch_box(uint32_t to, const CUtensorMap* map, int col, int head, int row, int seq, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 :: "r"(to), "l"(map), "r"(col), "r"(head), "r"(row), "r"(seq), "r"(bar) : "memory");
}
__device__ __forceinline__ void fetch_to_l2(const CUtensorMap* map, int col, int head, int row, int seq)
{
    asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" :: "l"(map), "r"(col), "r"(head), "r"(row), "r"(seq) : "memory");
}

// As umma::wait, but asleep for up to 20 us at a time: many warps wait at once here, and what they would issue meanwhile slows the others down.
__device__ __forceinline__ void await(uint32_t bar, uint32_t parity, volatile int* dead)
{
    for (int i = 0; i < (1 << 16); ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
        if (ok)
            return;
        if ((i & 15) == 15 && *dead)
            return;
    }
    *dead = 1;
    g_error = 1;
}

// A warp's part in a barrier of all walking warps, behind what its lanes have written.
__device__ __forceinline__ void warp_arrives(uint32_t bar)
{
    __syncwarp();
    if (threadIdx.x % 32 == 0)
        arrive(bar);
}

// One piece and 64 value channels of one head, chunk by chunk.
//
// Every operand is read once from memory (queries and keys once for each 64 value channels), and nothing but the results is written: with the states of all chunks in memory
// between kernels for what a chunk adds, the states and the outputs, 4 x 2048 tokens of 16 heads of 128 x 128 took 97 us for three times the bytes.  Two warps load the
// next chunk's tiles and find its decays, one issues products, sixteen (512 threads) do the rest, each at its own pace:
//
//     values times exp(R_j), split        [U = k' (weighted values)]
//     scores times decays, q S_0 times exp(G_i)      [+ scores v]
//     S = exp(G_C) S + U, its image in 16 bits       [next q S_0]
//     (the next chunk's values), the results
//
// Tensor memory: scores, results of two chunks in turn, what the chunk adds to the state, and the weighted scores as an operand.
//
// Bounds: not memory (4 x 2048 tokens of 16 heads of 128 x 128 in 50 us, 2.8 TB/s) but a chunk's steps one behind the other, 4600 clocks: the products' operands take all of shared
// memory's bandwidth for 2600 of them, and the threads' instructions have to fit in between.
template <typename T, int DK>
__global__ void __launch_bounds__(kWalkBlock, 1) walk_kernel(const __grid_constant__ Maps maps, const AttnDev p)
{
    using S_ = WalkShape<T, DK>;
    using Small = typename S_::Small;
    constexpr int TERMS = S_::TERMS;
    char* smem = dattn_tiles;
    Small& sm = *reinterpret_cast<Small*>(smem + S_::TILES);
    const int splits = (p.dv + kCols - 1) / kCols;
    const Place where = place_of(p, splits);
    const int head = where.head, group = head / p.share, col0 = where.part * kCols;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int cols = min(kCols, p.dv - col0);
    wait_for_previous();
    const Piece piece = piece_at(p, where.piece);
    if (piece.owner < 0)
        return;
    const int n = __shfl_sync(0xffffffffu, (int)((piece.len + kChunk - 1) / kChunk), 0);
    if (threadIdx.x == 0) {
        auto init = [](uint64_t& bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(&bar)), "r"(count) : "memory"); };
        for (int i = 0; i < 2; ++i) {
            init(sm.loaded[i], 32 * kFrontWarps);
            init(sm.freed[i], kWalkWarps);
        }
        init(sm.scores, 1), init(sm.state, 1), init(sm.added, 1), init(sm.out, 1), init(sm.drained, 1);
        init(sm.weighted, kWalkWarps), init(sm.weighed, kWalkWarps), init(sm.imaged, kWalkWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.dead = 0;
    }
    if (warp == kWalkWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&sm.tmem)), "r"(S_::COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    before_barrier();
    __syncthreads();
    behind_barrier();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem, 0);
    const uint32_t tiles = __shfl_sync(0xffffffffu, smem_u32(smem), 0), weighted = tiles + 2 * S_::STAGE, image = weighted + TERMS * S_::V_BYTES;
    // tensor memory: what the chunk adds to the state (64 columns for each term), the weighted scores as an operand, results of two chunks in turn, scores
    const uint32_t added = tmem, operand = tmem + 192, scores = tmem + 384;
    auto keys_at = [&](int i) { return tiles + (i & 1) * S_::STAGE; };
    auto values_at = [&](int i) { return tiles + (i & 1) * S_::STAGE + S_::K_BYTES; };
    auto queries_at = [&](int i) { return tiles + (i & 1) * S_::STAGE + S_::K_BYTES + S_::V_BYTES; };
    auto results_at = [&](int i) { return tmem + 256 + (i & 1) * 64; };
    auto until = [&](uint64_t& bar, int phase) {
        await(smem_u32(&bar), phase & 1, &sm.dead);
        __syncwarp();
    };

    if (warp > kWalkWarps) {                     // ---- tiles and decays
        const int thread = threadIdx.x - 32 * (kWalkWarps + 1);
        const float A = rate(p, head), bias = p.delta.ptr && p.delta_bias ? p.delta_bias[head] : 0.f;
        T raw[4 / kFrontWarps];
        auto ask = [&](int i) {
            const Chunk c = chunk_of(piece, i);
#pragma unroll
            for (int b = 0; b < 4 / kFrontWarps; ++b) {
                const int t = b * 32 * kFrontWarps + thread;
                raw[b] = load_if(row_ptr<T>(p.delta, c.seq, c.row0 + t) + head, p.delta.ptr && t < c.len);
            }
        };
        if (n > 0)
            ask(0);
        for (int i = 0; i < n; ++i) {
            const Chunk c = chunk_of(piece, i);
            // by the copy engine, which fills up with zeros behind the matrix; the last chunk of a packed sequence, which others' rows follow, by the threads
            const bool engine = !p.seqs.offsets || c.len == kChunk;
            const uint32_t bar = smem_u32(&sm.loaded[i & 1]);
            bool arrived = false;
            auto fetch = [&]() {
                until(sm.freed[i & 1], i / 2 + 1);                   // passes at once for the first two
                if (engine) {
                    if (warp == kWalkWarps + 1) {
                        arrived = elect_one();
                        if (arrived) {
                            expect_bytes(bar, S_::STAGE);
                            const int row0 = (int)c.row0, seq = (int)c.seq;
                            fetch_box(values_at(i), &maps.v, col0, head, row0, seq, bar);
#pragma unroll
                            for (int b = 0; b < DK / 64; ++b)
                                fetch_box(keys_at(i) + b * kBox, &maps.k, b * 64, group, row0, seq, bar);
#pragma unroll
                            for (int b = 0; b < DK / 64; ++b)
                                fetch_box(queries_at(i) + b * kBox, &maps.q, b * 64, group, row0, seq, bar);
                            if (i + 2 < n) {                         // stages are free late: by then their next tiles have come half of the way
                                const int next = row0 + 2 * kChunk;
                                fetch_to_l2(&maps.v, col0, head, next, seq);
#pragma unroll
                                for (int b = 0; b < DK / 64; ++b) {
                                    fetch_to_l2(&maps.k, b * 64, group, next, seq);
                                    fetch_to_l2(&maps.q, b * 64, group, next, seq);
                                }
                            }
                        }
                        __syncwarp();
                    }
                } else {
                    load_tile<T, kCols, 32 * kFrontWarps>(values_at(i), p.v, c, head * p.head_v + col0, cols, thread);
                    load_tile<T, DK, 32 * kFrontWarps>(keys_at(i), p.k, c, group * p.head_k, p.dk, thread);
                    load_tile<T, DK, 32 * kFrontWarps>(queries_at(i), p.q, c, group * p.head_q, p.dk, thread);
                    copies_begun();
                }
            };
            if (i < 2)                           // nothing to wait for
                fetch();
            float sum[4 / kFrontWarps], behind[4 / kFrontWarps], low[4 / kFrontWarps];
#pragma unroll
            for (int b = 0; b < 4 / kFrontWarps; ++b) {
                const float l = log_decay(A, p.delta.ptr ? step_of(p, to_f(raw[b]) + bias) : 1.f);
                sum[b] = block_sums<!kIsBf16<T>>(b * 32 * kFrontWarps + thread < c.len ? l : 0.f, behind[b], low[b]);
                behind[b] = ex2(behind[b]);
            }
            if (i + 1 < n)
                ask(i + 1);
            if (i >= 2)
                fetch();
            Table& dec = sm.dec[i & 1];
#pragma unroll
            for (int b = 0; b < 4 / kFrontWarps; ++b) {
                const int t = b * 32 * kFrontWarps + thread;
                dec.g[t] = sum[b];
                if (!kIsBf16<T>)
                    sm.low[i & 1][t] = low[b];
                dec.to_end[t] = behind[b];
                if (lane == 31)
                    dec.block[t / 32] = sum[b];
            }
            asm volatile("bar.sync 2, %0;" :: "n"(32 * kFrontWarps) : "memory");
            if (thread < 12) {                   // before, behind, skipped, whole
                const float b0 = dec.block[0], b1 = dec.block[1], b2 = dec.block[2], b3 = dec.block[3];
                const int k = thread % 4;
                float e;
                if (thread < 4)
                    e = k == 0 ? 0.f : k == 1 ? b0 : k == 2 ? b0 + b1 : b0 + b1 + b2;
                else if (thread < 8)
                    e = k == 0 ? b1 + b2 + b3 : k == 1 ? b2 + b3 : k == 2 ? b3 : 0.f;
                else
                    e = k == 0 ? b1 : k == 1 ? b1 + b2 : k == 2 ? b2 : (b0 + b1) + (b2 + b3);
                (thread < 4 ? dec.before[k] : thread < 8 ? dec.behind[k] : k < 3 ? dec.skipped[k] : dec.whole) = ex2(e);
            }
            if (!engine) {
                copies_done<0>();
                to_tensor_cores();
            }
            __syncwarp();                        // what the elected lane wrote of the table, whose arrival came with its copies, is there before the others arrive
            if (!arrived)
                arrive(bar);
        }
        if (sm.dead) {                           // copies under way end before the block does
            for (int i = n > 2 ? n - 2 : 0; i < n; ++i)
                drain(smem_u32(&sm.loaded[i & 1]), i / 2 & 1);
        }
    } else if (warp == kWalkWarps) {             // ---- products
        auto score_products = [&](int i) {
            behind_barrier();
            constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, 128);
            if (elect_one()) {
                products<DK / 16, kColumns, kColumns>(scores, over_columns(queries_at(i), 0), over_columns(keys_at(i), 0), id, false);
                commit(smem_u32(&sm.scores));
            }
            __syncwarp();
        };
        if (n > 0) {
            until(sm.loaded[0], 0);
            score_products(0);
        }
        for (int i = 0; i < n; ++i) {
            until(sm.imaged, i);
            behind_barrier();
            constexpr uint32_t id = instruction(kIsBf16<T>, false, true, 128, kCols);
            const uint32_t to = results_at(i);
            if (elect_one()) {
                products<DK / 16, kColumns, 16>(to, over_columns(queries_at(i), 0), image_over_dk<DK>(image, 0), id, false);
                commit(smem_u32(&sm.state));
            }
            __syncwarp();
            until(sm.weighted, i);
            behind_barrier();
            {
                constexpr uint32_t id_added = instruction(kIsBf16<T>, true, true, 128, TERMS * kCols); // all terms beside one another: the keys are read once
                if (elect_one()) {
                    products<8, kTokens, kTokens>(added, over_tokens(keys_at(i), 0), over_tokens(weighted, 0), id_added, false);
                    commit(smem_u32(&sm.added));
                }
                __syncwarp();
            }
            until(sm.weighed, i);
            behind_barrier();
            if (elect_one()) {
                products_tmem<8, kTokens>(to, operand, over_tokens(values_at(i), 0), id);
                commit(smem_u32(&sm.out));
            }
            __syncwarp();
            if (i + 1 < n) {
                until(sm.loaded[(i + 1) & 1], (i + 1) / 2);
                score_products(i + 1);
            }
        }
        if (sm.dead) {                           // products under way end before tensor memory is given back
            if (elect_one())
                commit(smem_u32(&sm.drained));
            __syncwarp();
            drain(smem_u32(&sm.drained), 0);
        }
    } else {                                     // ---- everything else
        const int quarter = warp % 4, sub = warp / 4, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const long long place = ((where.piece * p.heads + head) * splits + where.part) * (kWalkThreads * 16);
        float S[16];
        if (!piece.first || !piece.last) {       // (the first piece too: the last one may write over the states in front of the sequences)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<float4*>(S + 4 * j) = *reinterpret_cast<const float4*>(p.piece_state + place + (j * kWalkThreads + threadIdx.x) * 4);
        } else {
            load_state(S, p, p.state, piece.owner, head, row, col0 + sub * 16);
        }
        float unit = 1.f, unit_v = 1.f, unit_row = 1.f;
        // the image of the state in 16 bits, [8 groups of 8 columns][DK rows]; float16: times a power of two, so that it neither overflows nor vanishes
        auto put_image = [&]() {
            float up = 1.f;
            if (!kIsBf16<T>) {
                float most = 0.f;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    most = fmaxf(most, fabsf(S[j]));
                up = power_for(walk_largest(quarter * 32 < DK ? most : 0.f, sm.most), unit);
            }
            if (quarter * 32 < DK) {
#pragma unroll
                for (int j = 0; j < 16; j += 8) {
                    const uint4 w = make_uint4(pack16<T>(S[j] * up, S[j + 1] * up), pack16<T>(S[j + 2] * up, S[j + 3] * up), pack16<T>(S[j + 4] * up, S[j + 5] * up),
                                               pack16<T>(S[j + 6] * up, S[j + 7] * up));
                    *reinterpret_cast<uint4*>(smem + (image - tiles) + ((sub * 2 + j / 8) * DK + row) * 16) = w;
                }
            }
            to_tensor_cores();
            before_barrier();
            warp_arrives(smem_u32(&sm.imaged));
        };
        // values times their decays to the chunk's end, split
        auto put_values = [&](int i) {
            until(sm.loaded[i & 1], i / 2);
            uint4 v[2];
            float up = 1.f, most = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = h * kWalkThreads + threadIdx.x;
                v[h] = *reinterpret_cast<const uint4*>(smem + (values_at(i) - tiles) + tile_at(e / 8, e % 8));
                if (!kIsBf16<T>) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 x = unpack16<T>((&v[h].x)[j]);
                        most = fmaxf(most, fmaxf(fabsf(x.x), fabsf(x.y)));
                    }
                }
            }
            if (!kIsBf16<T>)
                up = power_for(walk_largest(most, sm.most + kWalkWarps), unit_v);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = h * kWalkThreads + threadIdx.x;
                const Table& dec = sm.dec[i & 1];
                const float w = dec.to_end[e / 8] * (dec.behind[e / 256] * up);
                uint4 term[TERMS];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    split_terms<T, TERMS>((&v[h].x)[j], w, [&](int t, uint32_t u) { (&term[t].x)[j] = u; });
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
                    *reinterpret_cast<uint4*>(smem + (weighted - tiles) + t * S_::V_BYTES + tile_at(e / 8, e % 8)) = term[t];
            }
            to_tensor_cores();
            before_barrier();
            warp_arrives(smem_u32(&sm.weighted));
        };
        // scores times decays, q S_0 times exp(G_i), the state behind the chunk
        auto weigh = [&](int i) {
            const Table& dec = sm.dec[i & 1];
            const float across = dec.whole;
            const float mine = dec.g[row], own = ex2(mine) * p.scale;
            float f = own * dec.before[quarter];
            until(sm.scores, i);
            behind_barrier();
            // a warp has one of the earlier blocks of 32 tokens and a quarter of its rows' own block, where the exponentials are (all of that in one warp took
            // 1700 clocks of a chunk's 4600; the later blocks are zeros)
            uint32_t packed[16], own_block[4];
            float most = 0.f, most_own = 0.f, over = 0.f, over_own = 0.f;           // (nothing is changed into nothing)
            if (sub < quarter) {
                float v[32];
                tmem_ld32(scores + sub * 32 + lanes, v);
                decay_earlier(v, own * between(dec, sub, quarter), dec.to_end + sub * 32);
                pack_weights<T>(v, packed, most, over);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    packed[j] = 0;
            }
            {
                const int at = quarter * 32 + sub * 8;
                float v[8];
                tmem_ld8(scores + at + lanes, v);
                const float* low = sm.low[i & 1];
                const float mine_low = kIsBf16<T> ? 0.f : low[row];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {                     // (of later tokens it may be infinite: they are taken out behind it)
                    const float2 h = *reinterpret_cast<const float2*>(dec.g + at + j);
                    float d0 = mine - h.x, d1 = mine - h.y;
                    if (!kIsBf16<T>) {
                        const float2 l = *reinterpret_cast<const float2*>(low + at + j);
                        d0 += mine_low - l.x, d1 += mine_low - l.y;
                    }
                    v[j] *= p.scale * ex2(d0), v[j + 1] *= p.scale * ex2(d1);
                    if (!kIsBf16<T>) {
                        v[j] = lane >= sub * 8 + j ? v[j] : 0.f;
                        v[j + 1] = lane > sub * 8 + j ? v[j + 1] : 0.f;
                    }
                }
                pack_weights<T>(v, own_block, most_own, over_own);
                if (kIsBf16<T>) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2)
                        own_block[j / 2] = lane > sub * 8 + j ? own_block[j / 2] : lane == sub * 8 + j ? own_block[j / 2] & 0xffffu : 0u;
                }
            }
            if (kIsBf16<T>) {
                f *= unit;
            } else {                             // the power of the four warps that share the row
                sm.row_most[sub][row] = fmaxf(most, most_own);
                asm volatile("bar.sync %0, 128;" :: "r"(3 + quarter) : "memory");
                const float up = row_power(fmaxf(fmaxf(sm.row_most[0][row], sm.row_most[1][row]), fmaxf(sm.row_most[2][row], sm.row_most[3][row])), highest_with(unit), unit_row);
                change_power(packed, up * over);
                change_power(own_block, up * over_own);
                f *= unit * up;
            }
            if (sub != quarter)
                tmem_st16(operand + sub * 16 + lanes, packed);
            tmem_st4(operand + quarter * 16 + sub * 4 + lanes, own_block);
            until(sm.state, i);
            behind_barrier();
            float v[16];
            tmem_ld16(results_at(i) + sub * 16 + lanes, v);
            scale_all(v, f);
            tmem_st16(results_at(i) + sub * 16 + lanes, reinterpret_cast<const uint32_t(&)[16]>(v));
            tmem_st_done();
            before_barrier();
            warp_arrives(smem_u32(&sm.weighed));
            until(sm.added, i);
            behind_barrier();
            if (quarter * 32 < DK) {
                float u[16];
                tmem_ld16(added + (TERMS - 1) * kCols + sub * 16 + lanes, u);
#pragma unroll
                for (int t = TERMS - 2; t >= 0; --t) {
                    float v[16];
                    tmem_ld16(added + t * kCols + sub * 16 + lanes, v);
                    add_all(u, v);
                }
                if (!kIsBf16<T>)
                    scale_all(u, unit_v);
                carry_all(S, across, u);
            }
        };
        // (the products' sum) to memory
        auto put_results = [&](int i) {
            const Chunk c = chunk_of(piece, i);
            float v[16];
            until(sm.out, i);
            behind_barrier();
            tmem_ld16(results_at(i) + sub * 16 + lanes, v);
            if (!kIsBf16<T>)
                scale_all(v, unit_row);
            // through the place of the values, which are done with, so that rows are written as a whole
            char* stage = smem + (values_at(i) - tiles);
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
                const uint4 w = make_uint4(pack16<T>(v[j], v[j + 1]), pack16<T>(v[j + 2], v[j + 3]), pack16<T>(v[j + 4], v[j + 5]), pack16<T>(v[j + 6], v[j + 7]));
                *reinterpret_cast<uint4*>(stage + tile_at(row, sub * 2 + j / 8)) = w;
            }
            asm volatile("bar.sync %0, 128;" :: "r"(3 + quarter) : "memory");          // the four warps of these rows
            T* to = row_ptr<T>(p.y, c.seq, c.row0 + quarter * 32) + (long long)head * p.dv + col0;
            if (p.vec_y == 16) {
                uint4 w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int e = h * 128 + sub * 32 + lane;
                    w[h] = *reinterpret_cast<const uint4*>(stage + tile_at(quarter * 32 + e / 8, e % 8));
                }
                to_tensor_cores();           // (with stores to memory under way this would wait for them)
                before_barrier();
                warp_arrives(smem_u32(&sm.freed[i & 1]));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int e = h * 128 + sub * 32 + lane, r = e / 8, c8 = e % 8;
                    if (quarter * 32 + r < c.len && c8 * 8 < cols)
                        *reinterpret_cast<uint4*>(to + r * p.y.ts + c8 * 8) = w[h];
                }
            } else {
                if (p.vec_y == 8) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int e = h * 128 + sub * 32 + lane, r = e / 16, c4 = e % 16;
                        if (quarter * 32 + r < c.len && c4 * 4 < cols)
                            *reinterpret_cast<uint2*>(to + r * p.y.ts + c4 * 4) = *reinterpret_cast<const uint2*>(stage + tile_at(quarter * 32 + r, c4 / 2) + c4 % 2 * 8);
                    }
                } else {
                    for (int e = sub * 32 + lane; e < 32 * kCols; e += 128) {
                        const int r = e / kCols, k = e % kCols;
                        if (quarter * 32 + r < c.len && k < cols)
                            to[r * p.y.ts + k] = reinterpret_cast<const T*>(stage + tile_at(quarter * 32 + r, k / 8))[k % 8];
                    }
                }
                to_tensor_cores();
                before_barrier();
                warp_arrives(smem_u32(&sm.freed[i & 1]));
            }
        };
        for (int i = -1; i < n; ++i) {           // (what is made for the next chunk has its code once: the first passes through it wait for instructions)
            if (i >= 0)
                weigh(i);
            if (i + 1 < n) {
                put_image();
                put_values(i + 1);
            }
            if (i >= 0)
                put_results(i);
        }
        if (piece.last)
            store_state(S, p, p.state_out, piece.owner, head, row, col0 + sub * 16);
    }
    before_barrier();
    __syncthreads();
    if (warp == kWalkWarps)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(S_::COLUMNS) : "memory");
}

// ---- states alone ---------------------------------------------------------------------------------------------------------

// What a state walk does: along a sequence or, `back`, from its end (with queries for keys and the gradients of y for values: the gradients of the states), for what a piece adds,
// from zero, or for the states in front of all chunks.
struct StateDev {
    Rows k, v;
    int head_k, head_v, back;
    const float* given;                          // in front of the sequences (back: behind them)
    float* last;                                 // behind them (in front)
    float factor;                                // of what is added
    float *piece_state, *piece_decay;            // of the pieces of a sequence, as the threads of a walk have them: what each adds, then the state in front of it; [pieces][heads]
    // the states in front of the chunks in 16 bits, [chunks][heads][terms][DV / 8][DK][8], as sums of two numbers or three; float16: what they have to be multiplied by
    char* image;
    float* unit;
    int image_bytes, terms;
    // back: <Z, S_0> exp(G_C) of every chunk from the images of S_0: the shares of the warps of its walks, [chunks][heads][splits][16]
    const char* other;
    const float* other_unit;
    float* across;
    float* whole;                                // or exp(G_C) alone, for a kernel of its own, [chunks][heads]
};
// Walks of one launch: one along the sequences, or one each way.
struct States {
    StateDev way[2];
    int ways;
    const int* seq_first;                        // packed sequences: the first chunk of each
};

template <typename T, int DK, int COLS> struct StateShape {
    static constexpr int TERMS = kIsBf16<T> ? 3 : 2;
    static constexpr int K_BYTES = DK / 64 * kBox, V_BYTES = COLS / 64 * kBox, STAGE = K_BYTES + V_BYTES;
    struct alignas(16) Weights {
        float own[kChunk];                       // of each token, within its block of 32
        float block[4], of_block[4];             // sums over the blocks; weights of whole blocks
        float whole;
    };
    struct Small {
        uint64_t loaded[2], freed[2], weighted[2], added[2], drained;                // of chunks in turn
        uint32_t tmem;
        int dead;
        Weights dec[2];
        float most[3][kWalkWarps];               // of values of chunks in turn, of the state
    };
    // weighted values of two chunks, where there is room, and their products: the next ones are made while a chunk's products run
    static constexpr int TURNS = 2 * STAGE + 2 * TERMS * V_BYTES <= 225 * 1024 ? 2 : 1;
    static constexpr int TILES = 2 * STAGE + TURNS * TERMS * V_BYTES;
    static constexpr int SMEM = TILES + sizeof(Small);
    static constexpr int COLUMNS = TURNS * TERMS * COLS > 256 ? 512 : 256;
};
static_assert(StateShape<bf16, 128, 128>::SMEM <= 232448, "shared memory of a block");

// One piece of one head (COLS value channels of it), chunk by chunk: values times their weights, split into TERMS numbers of 16 bits, all terms beside one another as one operand of the
// product with the keys; the state in registers, COLS / 4 neighbouring columns of a row of dk to a thread.  Warps have the roles of walk_kernel's.  4 x 1024 tokens of 16 heads of
// 128 x 128, images in three terms: 28 us each way (48 KB read and written for each chunk and 64 columns, 3.6 TB/s).
template <typename T, int DK, int COLS>
__global__ void __launch_bounds__(kWalkBlock, 1) state_walk_kernel(const __grid_constant__ Maps maps_there, const __grid_constant__ Maps maps_back, const AttnDev p, const States states,
                                                                   int splits)
{
    const Place where = place_of(p, splits * states.ways);
    const StateDev& q = states.way[where.part / splits];
    const Maps& maps = where.part / splits ? maps_back : maps_there;
    const int z = where.part % splits;
    const bool BACK = q.back;
    using S_ = StateShape<T, DK, COLS>;
    using Small = typename S_::Small;
    constexpr int TERMS = S_::TERMS, OWN = COLS / 4;
    char* smem = dattn_tiles;
    Small& sm = *reinterpret_cast<Small*>(smem + S_::TILES);
    const int head = where.head, group = head / p.share, col0 = z * COLS;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int cols = min(COLS, p.dv - col0);
    wait_for_previous();
    const Piece piece = piece_at(p, where.piece);
    if (piece.owner < 0 || (!q.image && (BACK ? piece.first : piece.last)))
        return;
    // its first chunk's number; offsets that decrease could ask for more chunks than there is room for: those behind are left out
    const long long first = q.image ? (p.seqs.offsets ? states.seq_first[piece.owner] : piece.owner * p.chunks_per_seq) + piece.t0 / kChunk : 0;
    const long long chunks = (piece.len + kChunk - 1) / kChunk;
    const int n = __shfl_sync(0xffffffffu, (int)(q.image ? min(chunks, max(p.chunks - first, 0ll)) : chunks), 0);
    if (threadIdx.x == 0) {
        auto init = [](uint64_t& bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(&bar)), "r"(count) : "memory"); };
        for (int i = 0; i < 2; ++i) {
            init(sm.loaded[i], 32 * kFrontWarps);
            init(sm.freed[i], kWalkWarps);
            init(sm.weighted[i], kWalkWarps);
            init(sm.added[i], 1);
        }
        init(sm.drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.dead = 0;
    }
    if (warp == kWalkWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&sm.tmem)), "r"(S_::COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    before_barrier();
    __syncthreads();
    behind_barrier();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem, 0);
    const uint32_t tiles = __shfl_sync(0xffffffffu, smem_u32(smem), 0), weighted = tiles + 2 * S_::STAGE;
    auto keys_at = [&](int i) { return tiles + (i & 1) * S_::STAGE; };
    auto values_at = [&](int i) { return tiles + (i & 1) * S_::STAGE + S_::K_BYTES; };
    auto until = [&](uint64_t& bar, int phase) {
        await(smem_u32(&bar), phase & 1, &sm.dead);
        __syncwarp();
    };
    auto chunk = [&](int i) { return BACK ? n - 1 - i : i; };

    if (warp > kWalkWarps) {                     // ---- tiles and decays
        const int thread = threadIdx.x - 32 * (kWalkWarps + 1);
        const float A = rate(p, head), bias = p.delta.ptr && p.delta_bias ? p.delta_bias[head] : 0.f;
        T raw[4 / kFrontWarps];
        auto ask = [&](int i) {
            const Chunk c = chunk_of(piece, chunk(i));
#pragma unroll
            for (int b = 0; b < 4 / kFrontWarps; ++b) {
                const int t = b * 32 * kFrontWarps + thread;
                raw[b] = load_if(row_ptr<T>(p.delta, c.seq, c.row0 + t) + head, p.delta.ptr && t < c.len);
            }
        };
        if (n > 0)
            ask(0);
        for (int i = 0; i < n; ++i) {
            const Chunk c = chunk_of(piece, chunk(i));
            const bool engine = !p.seqs.offsets || c.len == kChunk;
            const uint32_t bar = smem_u32(&sm.loaded[i & 1]);
            bool arrived = false;
            float sum[4 / kFrontWarps], own[4 / kFrontWarps];
            auto find = [&]() {
#pragma unroll
                for (int b = 0; b < 4 / kFrontWarps; ++b) {
                    const float l = log_decay(A, p.delta.ptr ? step_of(p, to_f(raw[b]) + bias) : 1.f);
                    float behind, low;           // (no differences here)
                    sum[b] = block_sums<false>(b * 32 * kFrontWarps + thread < c.len ? l : 0.f, behind, low);
                    own[b] = ex2(BACK ? sum[b] : behind);
                }
                if (i + 1 < n)
                    ask(i + 1);
            };
            if (i >= 2)                          // while there is no room for the tiles
                find();
            until(sm.freed[i & 1], i / 2 + 1);
            if (engine) {
                if (warp == kWalkWarps + 1) {
                    arrived = elect_one();
                    if (arrived) {
                        expect_bytes(bar, S_::STAGE);
                        const int row0 = (int)c.row0, seq = (int)c.seq;
#pragma unroll
                        for (int b = 0; b < COLS / 64; ++b)
                            fetch_box(values_at(i) + b * kBox, &maps.v, col0 + b * 64, head, row0, seq, bar);
#pragma unroll
                        for (int b = 0; b < DK / 64; ++b)
                            fetch_box(keys_at(i) + b * kBox, &maps.k, b * 64, group, row0, seq, bar);
                        if (i + 2 < n) {
                            const int next = BACK ? row0 - 2 * kChunk : row0 + 2 * kChunk;
#pragma unroll
                            for (int b = 0; b < COLS / 64; ++b)
                                fetch_to_l2(&maps.v, col0 + b * 64, head, next, seq);
#pragma unroll
                            for (int b = 0; b < DK / 64; ++b)
                                fetch_to_l2(&maps.k, b * 64, group, next, seq);
                        }
                    }
                    __syncwarp();
                }
            } else {
                load_tile<T, COLS, 32 * kFrontWarps>(values_at(i), q.v, c, head * q.head_v + col0, cols, thread);
                load_tile<T, DK, 32 * kFrontWarps>(keys_at(i), q.k, c, group * q.head_k, p.dk, thread);
                copies_begun();
            }
            if (i < 2)
                find();
            typename S_::Weights& dec = sm.dec[i & 1];
#pragma unroll
            for (int b = 0; b < 4 / kFrontWarps; ++b) {
                const int t = b * 32 * kFrontWarps + thread;
                dec.own[t] = own[b];
                if (lane == 31)
                    dec.block[t / 32] = sum[b];
            }
            asm volatile("bar.sync 2, %0;" :: "n"(32 * kFrontWarps) : "memory");
            if (thread < 5) {
                const float b0 = dec.block[0], b1 = dec.block[1], b2 = dec.block[2], b3 = dec.block[3];
                const int k = BACK ? thread : 3 - thread;
                float e;
                if (BACK)
                    e = k == 0 ? 0.f : k == 1 ? b0 : k == 2 ? b0 + b1 : b0 + b1 + b2;
                else
                    e = k == 0 ? 0.f : k == 1 ? b3 : k == 2 ? b2 + b3 : b1 + b2 + b3;
                if (thread < 4)
                    dec.of_block[thread] = ex2(e);
                else
                    dec.whole = ex2((b0 + b1) + (b2 + b3));
            }
            if (!engine) {
                copies_done<0>();
                to_tensor_cores();
            }
            __syncwarp();                        // what the elected lane wrote of the table, whose arrival came with its copies, is there before the others arrive
            if (!arrived)
                arrive(bar);
        }
        if (sm.dead) {                           // copies under way end before the block does
            for (int i = n > 2 ? n - 2 : 0; i < n; ++i)
                drain(smem_u32(&sm.loaded[i & 1]), i / 2 & 1);
        }
    } else if (warp == kWalkWarps) {             // ---- products
        for (int i = 0; i < n; ++i) {
            until(sm.weighted[i & 1], i / 2);
            behind_barrier();
            constexpr int N = TERMS * COLS < 256 ? TERMS * COLS : 256, REST = TERMS * COLS - N;
            constexpr uint32_t id = instruction(kIsBf16<T>, true, true, 128, N);
            const uint64_t a = over_tokens(keys_at(i), 0), b = over_tokens(weighted + i % S_::TURNS * (TERMS * S_::V_BYTES), 0);
            const uint32_t to = tmem + i % S_::TURNS * (TERMS * COLS);
            if (elect_one()) {
#pragma unroll 1
                for (int s = 0; s < 8; ++s) {
                    mma(to, a + (s * 2048 >> 4), b + (s * 2048 >> 4), id, s > 0);
                    if constexpr (REST > 0)
                        mma(to + N, a + (s * 2048 >> 4), b + (N / 64 * kBox + s * 2048 >> 4), instruction(kIsBf16<T>, true, true, 128, REST), s > 0);
                }
                commit(smem_u32(&sm.added[i & 1]));
            }
            __syncwarp();
        }
        if (sm.dead) {                           // products under way end before tensor memory is given back
            if (elect_one())
                commit(smem_u32(&sm.drained));
            __syncwarp();
            drain(smem_u32(&sm.drained), 0);
        }
    } else {                                     // ---- everything else
        const int quarter = warp % 4, sub = warp / 4, row = quarter * 32 + lane;
        const bool mine = quarter * 32 < DK;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const long long place = ((where.piece * p.heads + head) * splits + z) * (kWalkThreads * OWN);
        float S[OWN];
        if (q.image && !(BACK ? piece.last : piece.first)) {
#pragma unroll
            for (int j = 0; j < OWN / 4; ++j)
                *reinterpret_cast<float4*>(S + 4 * j) = *reinterpret_cast<const float4*>(q.piece_state + place + (j * kWalkThreads + threadIdx.x) * 4);
        } else {
            load_state(S, p, q.image ? q.given : nullptr, piece.owner, head, row, col0 + sub * OWN);
        }
        float whole = 1.f;
        float unit_of[2] = {1.f, 1.f};
        // values times their weights, split
        auto put_values = [&](int i) {
            const typename S_::Weights& dec = sm.dec[i & 1];
            until(sm.loaded[i & 1], i / 2);
            float unit_v = 1.f;
            constexpr int VECTORS = COLS / 32;
            float up = 1.f;
            if (!kIsBf16<T>) {
                float most = 0.f;
#pragma unroll
                for (int h = 0; h < VECTORS; ++h) {
                    const int e = h * kWalkThreads + threadIdx.x, t = e / (COLS / 8);
                    const uint4 v = *reinterpret_cast<const uint4*>(smem + (values_at(i) - tiles) + tile_at(t, e % (COLS / 8)));
                    float here = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 x = unpack16<T>((&v.x)[j]);
                        here = fmaxf(here, fmaxf(fabsf(x.x), fabsf(x.y)));
                    }
                    most = fmaxf(most, here * (dec.own[t] * dec.of_block[t / 32]));
                }
                up = power_for(walk_largest(most, sm.most[i & 1]), unit_v);
            }
#pragma unroll
            for (int h = 0; h < VECTORS; ++h) {
                const int e = h * kWalkThreads + threadIdx.x, t = e / (COLS / 8);
                const uint32_t at = tile_at(t, e % (COLS / 8));
                const uint4 v = *reinterpret_cast<const uint4*>(smem + (values_at(i) - tiles) + at);
                const float w = dec.own[t] * (dec.of_block[t / 32] * up);
                uint4 term[TERMS];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    split_terms<T, TERMS>((&v.x)[j], w, [&](int n, uint32_t u) { (&term[n].x)[j] = u; });
#pragma unroll
                for (int n = 0; n < TERMS; ++n)
                    *reinterpret_cast<uint4*>(smem + (weighted - tiles) + (i % S_::TURNS * TERMS + n) * S_::V_BYTES + at) = term[n];
            }
            to_tensor_cores();
            before_barrier();
            warp_arrives(smem_u32(&sm.weighted[i & 1]));
            unit_of[i & 1] = unit_v;
        };
        for (int i = -1; i < n; ++i) {           // (what is made for the next chunk has its code once)
            if (i < 0) {
                if (n > 0)
                    put_values(0);
                continue;
            }
            const typename S_::Weights& dec = sm.dec[i & 1];
            uint4 other[OWN / 8][TERMS];         // asked for early
            const long long at = (first + chunk(i)) * p.heads + head;
            const long long place_of = at * ((long long)q.terms * q.image_bytes) + ((col0 + sub * OWN) / 8 * DK + row) * 16;
            if (q.other) {
#pragma unroll
                for (int j = 0; j < OWN / 8; ++j)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
                        other[j][t] = load_if(reinterpret_cast<const uint4*>(q.other + place_of + j * DK * 16 + t * q.image_bytes), mine && t < q.terms);
            }
            const float over = dec.whole;
            if (q.image) {                       // the state in front of the chunk, while the products run
                float up = 1.f;
                if (!kIsBf16<T>) {
                    float most = 0.f, unit;
#pragma unroll
                    for (int j = 0; j < OWN; ++j)
                        most = fmaxf(most, fabsf(S[j]));
                    up = power_for(walk_largest(mine ? most : 0.f, sm.most[2]), unit);
                    if (threadIdx.x == 0)
                        q.unit[at] = unit;
                }
                if (mine) {
#pragma unroll
                    for (int j = 0; j < OWN; j += 8) {
                        uint4 term[TERMS];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float x = S[j + 2 * k] * up, y = S[j + 2 * k + 1] * up;
#pragma unroll
                            for (int t = 0; t < TERMS; ++t) {
                                const uint32_t u = pack16<T>(x, y);
                                const float2 f = unpack16<T>(u);
                                (&term[t].x)[k] = u;
                                x -= f.x, y -= f.y;
                            }
                        }
                        char* to = q.image + place_of + j / 8 * DK * 16;
#pragma unroll
                        for (int t = 0; t < TERMS; ++t)
                            if (t < q.terms)
                                *reinterpret_cast<uint4*>(to + t * q.image_bytes) = term[t];
                    }
                }
                if (q.whole && threadIdx.x == 0 && z == 0)
                    q.whole[at] = over;
                if (q.other) {
                    float dot = 0.f;
#pragma unroll
                    for (int j = 0; j < OWN; j += 2) {
                        float2 f = make_float2(0.f, 0.f);
#pragma unroll
                        for (int t = TERMS - 1; t >= 0; --t) {
                            const float2 x = unpack16<T>((&other[j / 8][t].x)[j % 8 / 2]);
                            f.x += x.x, f.y += x.y;
                        }
                        dot = fmaf(S[j], f.x, dot);
                        dot = fmaf(S[j + 1], f.y, dot);
                    }
                    dot = mine ? dot : 0.f;
#pragma unroll
                    for (int o = 16; o; o /= 2)
                        dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    if (lane == 0)
                        q.across[(at * splits + z) * kWalkWarps + warp] = dot * over * (kIsBf16<T> ? 1.f : q.other_unit[at]);
                }
            }
            if (S_::TURNS == 2 && i + 1 < n)
                put_values(i + 1);
            until(sm.added[i & 1], i / 2);
            behind_barrier();
            const uint32_t from = tmem + i % S_::TURNS * (TERMS * COLS);
            const float unit_v = kIsBf16<T> ? 1.f : i & 1 ? unit_of[1] : unit_of[0];
            if (mine) {
#pragma unroll
                for (int j = 0; j < OWN; j += 16) {
                    float u[16];
                    tmem_ld16(from + (TERMS - 1) * COLS + sub * OWN + j + lanes, u);
#pragma unroll
                    for (int t = TERMS - 2; t >= 0; --t) {
                        float v[16];
                        tmem_ld16(from + t * COLS + sub * OWN + j + lanes, v);
                        add_all(u, v);
                    }
                    scale_all(u, unit_v * q.factor);
                    carry_all(reinterpret_cast<float(&)[16]>(S[j]), over, u);
                }
            }
            whole *= over;
            before_barrier();
            warp_arrives(smem_u32(&sm.freed[i & 1]));
            if (S_::TURNS == 1 && i + 1 < n)
                put_values(i + 1);
        }
        if (q.image) {
            if (BACK ? piece.first : piece.last)
                store_state(S, p, q.last, piece.owner, head, row, col0 + sub * OWN);
        } else {
            if (mine) {
#pragma unroll
                for (int j = 0; j < OWN / 4; ++j)
                    *reinterpret_cast<float4*>(q.piece_state + place + (j * kWalkThreads + threadIdx.x) * 4) = *reinterpret_cast<const float4*>(S + 4 * j);
            }
            if (threadIdx.x == 0 && z == 0)
                q.piece_decay[where.piece * p.heads + head] = whole;
        }
    }
    before_barrier();
    __syncthreads();
    if (warp == kWalkWarps)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(S_::COLUMNS) : "memory");
}

// The states in front of the pieces (BACK: behind them), from what each adds: S = exp(..) S + U along a sequence, eight pieces' loads under way together.  A block works for the
// sequence whose last piece its number is, and for four of the `own` columns that a thread has in a state walk.  18 pieces of 8 heads of 64 x 64: 9 us, three loads one behind the
// other and a launch.
static __global__ void __launch_bounds__(kWalkThreads) join_kernel(const AttnDev p, const States states, int own, int splits)
{
    constexpr int AHEAD = 8;
    wait_for_previous();
    const int parts = own / 4, head = blockIdx.y, z = blockIdx.z / parts % splits, part = blockIdx.z % parts;
    const StateDev& q = states.way[blockIdx.z / parts / splits];
    const bool back = q.back;
    long long first = p.seqs.offsets ? 0 : blockIdx.x / p.pieces_per_seq * p.pieces_per_seq;
    const Piece piece = piece_at(p, blockIdx.x, &first);
    const int lane = threadIdx.x % 32, quarter = threadIdx.x / 32 % 4, sub = threadIdx.x / 128, row = quarter * 32 + lane;
    if (piece.owner < 0 || !piece.last || piece.first || row >= (p.dk > 64 ? 128 : 64))        // (rows behind dk are zeros)
        return;
    const long long n = blockIdx.x - first + 1;
    float four[4];
    load_state(four, p, q.given, piece.owner, head, row, z * 4 * own + sub * own + part * 4);
    float4 S = make_float4(four[0], four[1], four[2], four[3]);
    auto which = [&](long long i) { return back ? first + n - 1 - i : first + i; };
    auto at = [&](long long i) {
        return reinterpret_cast<float4*>(q.piece_state + ((which(i) * p.heads + head) * splits + z) * (long long)(kWalkThreads * own)) + part * kWalkThreads + threadIdx.x;
    };
    for (long long i0 = 0; i0 < n - 1; i0 += AHEAD) {
        float4 u[AHEAD];
        float w[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const bool ok = i0 + i < n - 1;
            u[i] = load_if(at(ok ? i0 + i : 0), ok);
            w[i] = load_if(q.piece_decay + which(ok ? i0 + i : 0) * p.heads + head, ok);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (i0 + i < n - 1) {
                *at(i0 + i) = S;
                S.x = fmaf(w[i], S.x, u[i].x), S.y = fmaf(w[i], S.y, u[i].y), S.z = fmaf(w[i], S.z, u[i].z), S.w = fmaf(w[i], S.w, u[i].w);
            }
        }
    }
    *at(n - 1) = S;
}

// ---- one token of each sequence -------------------------------------------------------------------------------------------

constexpr int kStepThreads = 128;

// The state is read and written once, which is all that counts.  A block has all rows and COLS columns of a head's state: a thread 4 columns
// (V = 4; 1 where states cannot be accessed by 16 bytes) of every PARTS-th row, in loads of eight rows that are under way together.  67 MB of states in 26 us: read and written at 5.1 TB/s.
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
    const float a = ex2(rate(p, head) * d * kLog2e + kExBias);
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
