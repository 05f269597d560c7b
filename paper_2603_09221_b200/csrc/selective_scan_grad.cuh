// Gradients of the selective state space scan (selective_scan.cuh).  With g_t = dy_t silu(z_t) and the co-states
//     q_t = C_t g_t + exp(D_{t+1} A) q_{t+1}
// both recurrences, h forward and q backward, have the same decays, and the product of a span's decays is exp(A sum D_t).
// Every sequence is cut into pieces of 16 tokens:
//   1  local_kernel    of every piece, from nothing: the state behind it, the co-state a_{t0} q_{t0} in front of it (in the
//                      same walk: the running product of decays times C_t g_t) and the sum of its D_t
//   2  join_kernel     along every sequence: the state that enters each piece, the co-state that comes back to it; dstate
//   3  piece_kernel    of every piece, from those, in two halves of as many tokens as registers hold states for: states
//                      forward, co-states backward, every gradient
//   4  reduce kernels  the blocks' shares of dA, dD, ddelta_bias and of dB, dC, in a fixed order
// Steps 1 and 3 run over all tokens at once, whatever the number of sequences and channels.  A lane holds four states of two
// channels, as in the forward kernel.  Decays are computed again rather than kept, against 64 more registers and half the warps:
// 3.5 exponentials per state and token in all (one in step 1; in step 3 one for the states, a half for the first half's,
// which are walked twice, and one for the co-states).
//
// 4 sequences of 1024 tokens, 2048 channels, 16 states, bfloat16: 70 + 19 + 228 + 13 us; step 3 is bound by issue slots (49 %) and
// by the 11 warps of an SM (168 registers) that wait for one another's values.  Step 3 with decays kept, one channel to a lane:
// 555 us; computed again, two channels: 258; one copy of the code for both halves, which then fits the instruction cache: 239, now 228;
// with 128 registers (spills) 259; runs of eight pieces to a block instead of four 261 (fewer blocks in the last round).
#pragma once

#include "selective_scan.cuh"

namespace ttc {
namespace sscan {

constexpr int kGradThreads = 128;
constexpr int kPiece = 16, kHalfPiece = 8;     // tokens of a piece, and as many as a thread's registers hold states for
constexpr int kRun = 4;           // pieces that a block works through, one behind the other, with one share of dA and dD for all

struct GradDev {
    ScanDev f;                    // f.piece = kPiece * kRun: a run of pieces; run r holds the pieces r * kRun ..
    Rows dy, dx, ddelta, dB, dC, dz;
    const float* dstate_out;
    float *dA, *dD, *ddelta_bias, *dstate;
    long long runs;
    float *h, *r, *step;          // [runs * kRun][d][n] twice, [runs * kRun][d]
    float* part_A;                // [runs][d][n]
    float* part_D;                // [runs][2][d]: dD, ddelta_bias
    float* part_BC;               // [chan_blocks][runs * kRun * kPiece][groups][2][NP]
};

template <int LANES> struct Tile {
    static constexpr int CH = 2 * kGradThreads / LANES, NP = LANES * 4, TB = kPiece;
    static constexpr int WARPS = kGradThreads / 32;
    // floats: D, Dx of a channel pair; g of it; B; C
    static constexpr int TOK = TB * CH * 2, G = TB * CH, BC = TB * NP;
    // of half a piece: the lanes' shares of C . h, of q . B and A . (q a h); the warps' shares of dB and dC
    static constexpr int Y = kHalfPiece * CH * LANES, Q = 2 * Y, S = WARPS * kHalfPiece * 2 * NP;
    static constexpr size_t smem_local() { return sizeof(float) * (TOK + G + 2 * BC); }
    static constexpr size_t smem_piece() { return smem_local() + sizeof(float) * (Y + Q + S); }
};

// A piece's rows: loads under way in registers, then step sizes, D_t x_t, dy_t silu(z_t), B and C in shared memory.
template <typename T, int LANES, int V> struct Loader {
    using S = Tile<LANES>;
    static constexpr int CH = S::CH, NP = S::NP, TB = S::TB;
    static constexpr int COLS = CH / V, ROWS = kGradThreads / COLS, PASSES = (TB + ROWS - 1) / ROWS;
    static constexpr int BCOLS = NP / V, BROWS = kGradThreads / BCOLS, BPASSES = (TB + BROWS - 1) / BROWS;
    Vec<T, V> x[PASSES], delta[PASSES], dy[PASSES], z[PASSES], B[BPASSES], C[BPASSES];
    int lc, lr, chan, bc, br, group;
    bool mine, mine_b;
    float bias[V];

    __device__ __forceinline__ void start(const GradDev& p, int group_, int per_group, int c0)
    {
        const int tid = threadIdx.x;
        group = group_;
        lc = tid % COLS * V, lr = tid / COLS;
        chan = group * per_group + c0 + lc;
        mine = c0 + lc < per_group && lr < TB;
        bc = tid % BCOLS * V, br = tid / BCOLS;
        mine_b = bc < p.f.n && br < TB;
#pragma unroll
        for (int v = 0; v < V; ++v)
            bias[v] = p.f.delta_bias && mine ? p.f.delta_bias[chan + v] : 0.f;
    }
    __device__ __forceinline__ void rows(Vec<T, V> (&to)[PASSES], const Rows& r, long long seq, long long row, bool ok, int left)
    {
        const T* from = row_ptr<const T>(r, seq, row + lr) + chan;
        const long long pass = ROWS * r.ts;
#pragma unroll
        for (int e = 0; e < PASSES; ++e, from += pass)
            to[e] = load_if(reinterpret_cast<const Vec<T, V>*>(from), ok && lr + e * ROWS < left);
    }
    __device__ __forceinline__ void shared_rows(Vec<T, V> (&to)[BPASSES], const Rows& r, const GradDev& p, long long seq, long long row, int left)
    {
        const T* from = row_ptr<const T>(r, seq, row + br) + group * p.f.n + bc;
        const long long pass = BROWS * r.ts;
#pragma unroll
        for (int e = 0; e < BPASSES; ++e, from += pass)
            to[e] = load_if(reinterpret_cast<const Vec<T, V>*>(from), mine_b && br + e * BROWS < left);
    }
    // rows row .. row + left of the sequence (at most a piece)
    __device__ __forceinline__ void load(const GradDev& p, long long seq, long long row, int left)
    {
        left = left < TB ? left : TB;
        rows(delta, p.f.delta, seq, row, mine, left);
        rows(x, p.f.x, seq, row, mine, left);
        rows(dy, p.dy, seq, row, mine, left);
        rows(z, p.f.z, seq, row, mine && p.f.z.ptr, left);
        shared_rows(B, p.f.B, p, seq, row, left);
        shared_rows(C, p.f.C, p, seq, row, left);
    }
    __device__ __forceinline__ void stage(const GradDev& p, int left, float4* s_tok, float2* s_g, float* s_B, float* s_C) const
    {
        const bool gated = p.f.z.ptr;
        if (ROWS <= TB || lr < TB) {
#pragma unroll
            for (int e = 0; e < PASSES; ++e) {
                const int u = e * ROWS + lr;
                const bool none = u >= left;                         // padding: nothing decays, nothing is added
                float4* tok = s_tok + u * (CH / 2) + lc / 2;
                float2* to_g = s_g + u * (CH / 2) + lc / 2;
                if constexpr (V == 2) {
                    f2 step = add2(pack2(to_f(delta[e].v[0]), to_f(delta[e].v[1])), pack2(bias[0], bias[1]));
                    if (p.f.softplus)
                        step = softplus2(step);
                    f2 g = pack2(to_f(dy[e].v[0]), to_f(dy[e].v[1]));
                    if (gated)
                        g = mul2(g, silu2(pack2(to_f(z[e].v[0]), to_f(z[e].v[1]))));
                    const f2 in = mul2(step, pack2(to_f(x[e].v[0]), to_f(x[e].v[1])));
                    *reinterpret_cast<ulonglong2*>(tok) = none ? make_ulonglong2(0, 0) : make_ulonglong2(step, in);
                    *reinterpret_cast<f2*>(to_g) = none ? 0 : g;
                } else {
                    float step = to_f(delta[e].v[0]) + bias[0], g = to_f(dy[e].v[0]);
                    if (p.f.softplus)
                        step = softplus(step);
                    if (gated)
                        g *= silu(to_f(z[e].v[0]));
                    reinterpret_cast<float*>(tok)[lc % 2] = none ? 0.f : step;
                    reinterpret_cast<float*>(tok)[2 + lc % 2] = none ? 0.f : step * to_f(x[e].v[0]);
                    reinterpret_cast<float*>(to_g)[lc % 2] = none ? 0.f : g;
                }
            }
        }
        if (BROWS <= TB || br < TB) {
#pragma unroll
            for (int e = 0; e < BPASSES; ++e) {
                const int at = (e * BROWS + br) * NP + bc;
                float b[V], c[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    b[v] = to_f(B[e].v[v]), c[v] = to_f(C[e].v[v]);
                put<V>(s_B + at, b);
                put<V>(s_C + at, c);
            }
        }
    }
};

// A thread's four states of two channels: where they lie, and A log2(e) as pairs of channels.
struct Mine {
    long long at[2];              // of state n0 of either channel in a [d][n] array
    int count[2];                 // states of it that exist, 0 .. 4
    f2 A2[4];
    __device__ __forceinline__ void start(const GradDev& p, int group, int per_group, int c0, int pair, int n0)
    {
        float a[2][4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int ch = c0 + 2 * pair + c;
            at[c] = (long long)(group * per_group + ch) * p.f.n + n0;
            count[c] = ch < per_group ? max(0, min(4, p.f.n - n0)) : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[c][i] = i < count[c] ? exponent(p.f.A[at[c] + i]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            A2[i] = pack2(a[0][i], a[1][i]);
    }
    __device__ __forceinline__ void get(const float* from, f2 (&v)[4], bool vec) const
    {
        float w[2][4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (vec) {
                const float4 u = count[c] ? *reinterpret_cast<const float4*>(from + at[c]) : make_float4(0.f, 0.f, 0.f, 0.f);
                w[c][0] = u.x, w[c][1] = u.y, w[c][2] = u.z, w[c][3] = u.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[c][i] = i < count[c] ? from[at[c] + i] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = pack2(w[0][i], w[1][i]);
    }
    __device__ __forceinline__ void set(float* to, const f2 (&v)[4], bool vec) const
    {
        float w[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            unpack2(v[i], w[0][i], w[1][i]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (vec) {
                if (count[c])
                    *reinterpret_cast<float4*>(to + at[c]) = make_float4(w[c][0], w[c][1], w[c][2], w[c][3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < count[c])
                        to[at[c] + i] = w[c][i];
            }
        }
    }
};

// exp(D A) of a token
__device__ __forceinline__ void decays(f2 (&a)[4], const f2 (&A2)[4], f2 step)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float e0, e1;
        unpack2(fma2(A2[i], step, pack2(kExBias, kExBias)), e0, e1);
        a[i] = pack2(ex2(e0), ex2(e1));
    }
}
// h = a h + D x B
__device__ __forceinline__ void advance(f2 (&h)[4], const f2 (&a)[4], f2 in, const float4& b4)
{
    float in0, in1;
    unpack2(in, in0, in1);
    const float b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = fma2(a[i], h[i], pack2(in0 * b[i], in1 * b[i]));
}

template <typename T, int LANES, int V>
__global__ void __launch_bounds__(kGradThreads, 4) grad_local_kernel(const GradDev p)
{
    using S = Tile<LANES>;
    constexpr int CH = S::CH, TB = S::TB;
    extern __shared__ float4 smem[];
    float4* s_tok = smem;                                            // [TB][CH / 2]
    float2* s_g = reinterpret_cast<float2*>(s_tok + S::TOK / 4);     // [TB][CH / 2]
    float* s_B = reinterpret_cast<float*>(s_g + S::G / 2);           // [TB][NP]
    float* s_C = s_B + S::BC;

    Piece q;
    if (!find_piece(p.f, blockIdx.x, q))
        return;
    const int tid = threadIdx.x, sub = tid % LANES, pair = tid / LANES;
    const int group = blockIdx.y / p.f.chan_blocks, per_group = p.f.d / p.f.groups;
    const int c0 = (blockIdx.y % p.f.chan_blocks) * CH;
    Mine my;
    my.start(p, group, per_group, c0, pair, sub * 4);
    Loader<T, LANES, V> tile;
    tile.start(p, group, per_group, c0);
    const long long states = (long long)p.f.d * p.f.n;
    int left = static_cast<int>(q.t1 - q.t0);
    long long row = q.row0 + q.t0, slot = (long long)blockIdx.x * kRun;
    tile.load(p, q.seq, row, left);
    for (; left > 0; left -= kPiece, row += kPiece, ++slot) {
        tile.stage(p, left, s_tok, s_g, s_B, s_C);
        __syncthreads();
        tile.load(p, q.seq, row + kPiece, left - kPiece);
        f2 h[4] = {0, 0, 0, 0}, r[4] = {0, 0, 0, 0}, prod[4], total = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            prod[i] = pack2(1.f, 1.f);
#pragma unroll 4
        for (int u = 0; u < TB; ++u) {
            const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[u * (CH / 2) + pair];
            f2 a[4];
            decays(a, my.A2, tok.x);
            advance(h, a, tok.y, reinterpret_cast<const float4*>(s_B)[u * LANES + sub]);
            const float2 g = s_g[u * (CH / 2) + pair];
            const float4 c4 = reinterpret_cast<const float4*>(s_C)[u * LANES + sub];
            const float c[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                prod[i] = mul2(prod[i], a[i]);
                r[i] = fma2(prod[i], pack2(g.x * c[i], g.y * c[i]), r[i]);
            }
            total = add2(total, tok.x);
        }
        my.set(p.h + slot * states, h, p.f.vec4);
        my.set(p.r + slot * states, r, p.f.vec4);
        if (sub == 0) {
            float s[2];
            unpack2(total, s[0], s[1]);
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (my.count[c])
                    p.step[slot * p.f.d + group * per_group + c0 + 2 * pair + c] = s[c];
        }
        __syncthreads();
    }
}

// blockIdx.z 0: states forward, 1: co-states backward.  In: what each piece adds; out: what enters it.  V states of a channel
// to a thread (four where n is a multiple of four).
template <int V> __global__ void __launch_bounds__(128) grad_join_kernel(const GradDev p)
{
    wait_for_previous();
    const long long at = ((long long)blockIdx.y * 128 + threadIdx.x) * V, size = (long long)p.f.d * p.f.n;
    if (at >= size)
        return;
    typedef Vec<float, V> Some;
    const long long seq = blockIdx.x, c = at / p.f.n;
    const long long first = (p.f.piece_map ? p.f.seq_first[seq] : seq * p.f.pieces_per_seq) * kRun;
    const long long most = p.f.piece_map ? (p.f.seq_first[seq + 1] * (long long)kRun - first) : p.f.pieces_per_seq * kRun;
    long long count = (span_of(p.f.seqs, seq).len + kPiece - 1) / kPiece;
    count = count < most ? count : most;
    float a[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        a[i] = exponent(p.f.A[at + i]);
    constexpr int kAhead = 8;
    const bool back = blockIdx.z;
    const long long start = back ? first + count - 1 : first;
    float* v = (back ? p.r : p.h) + start * size + at;
    const float* s = p.step + start * p.f.d + c;
    const long long v_next = back ? -size : size, s_next = back ? -(long long)p.f.d : p.f.d;
    const float* from = back ? p.dstate_out : p.f.state;
    Some h;
#pragma unroll
    for (int i = 0; i < V; ++i)
        h.v[i] = from ? from[seq * size + at + i] : 0.f;
    auto piece = [&](Some add, float step) {
        *reinterpret_cast<Some*>(v) = h;
        v += v_next;
#pragma unroll
        for (int i = 0; i < V; ++i)
            h.v[i] = fmaf(ex2(a[i] * step), h.v[i], add.v[i]);
    };
    for (; count >= kAhead; count -= kAhead) {
        Some add[kAhead];
        float step[kAhead];
        const float* vv = v;
#pragma unroll
        for (int i = 0; i < kAhead; ++i, vv += v_next, s += s_next)
            add[i] = *reinterpret_cast<const Some*>(vv), step[i] = *s;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            piece(add[i], step[i]);
    }
    for (; count > 0; --count, s += s_next)
        piece(*reinterpret_cast<const Some*>(v), *s);
    if (back && p.dstate)
#pragma unroll
        for (int i = 0; i < V; ++i)
            p.dstate[seq * size + at + i] = h.v[i];
}

template <typename T, int LANES, int V>
__global__ void __launch_bounds__(kGradThreads, 3) grad_piece_kernel(const GradDev p)
{
    using S = Tile<LANES>;
    using L = Loader<T, LANES, V>;
    constexpr int CH = S::CH, NP = S::NP, WARPS = S::WARPS, HALF = kHalfPiece;
    extern __shared__ float4 smem[];
    float4* s_tok = smem;                                            // [TB][CH / 2]
    float2* s_g = reinterpret_cast<float2*>(s_tok + S::TOK / 4);     // [TB][CH / 2]
    float* s_B = reinterpret_cast<float*>(s_g + S::G / 2);           // [TB][NP]
    float* s_C = s_B + S::BC;
    float4* s_q = reinterpret_cast<float4*>(s_C + S::BC);            // [HALF][CH / 2][LANES]: q . B and A . (q a h), of two channels
    float2* s_y = reinterpret_cast<float2*>(s_q + S::Q / 4);         // [HALF][CH / 2][LANES]: C . h
    float* s_BC = reinterpret_cast<float*>(s_y + S::Y / 2);          // [WARPS][HALF][2][NP]

    Piece q;
    if (!find_piece(p.f, blockIdx.x, q))
        return;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, sub = tid % LANES, pair = tid / LANES, n0 = sub * 4;
    const int group = blockIdx.y / p.f.chan_blocks, per_group = p.f.d / p.f.groups, block = blockIdx.y % p.f.chan_blocks;
    const int c0 = block * CH;
    Mine my;
    my.start(p, group, per_group, c0, pair, n0);
    L tile;
    tile.start(p, group, per_group, c0);
    float skip[V], sum_D[V] = {}, sum_bias[V] = {};
#pragma unroll
    for (int v = 0; v < V; ++v)
        skip[v] = p.f.D && tile.mine ? p.f.D[tile.chan + v] : 0.f;
    f2 dA[4] = {0, 0, 0, 0};
    const long long states = (long long)p.f.d * p.f.n;
    const bool want_z = p.dz.ptr;
    int left = static_cast<int>(q.t1 - q.t0);
    long long row = q.row0 + q.t0, slot = (long long)blockIdx.x * kRun;
    for (; left > 0; left -= kPiece, row += kPiece, ++slot) {
        tile.load(p, q.seq, row, left);
        f2 h0[4], h1[4], r[4];                                       // states in front of both halves, co-state behind
        my.get(p.h + slot * states, h0, p.f.vec4);
        my.get(p.r + slot * states, r, p.f.vec4);
        tile.stage(p, left, s_tok, s_g, s_B, s_C);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            h1[i] = h0[i];
#pragma unroll 4
        for (int u = 0; u < HALF; ++u) {
            const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[u * (CH / 2) + pair];
            f2 a[4];
            decays(a, my.A2, tok.x);
            advance(h1, a, tok.y, reinterpret_cast<const float4*>(s_B)[u * LANES + sub]);
        }
#pragma unroll 1
        for (int half = 1; half >= 0; --half) {                      // (one copy of the code: two overflow the instruction cache)
            if (half * HALF < left) {
                // states of the half, h[u] in front of token u
                f2 h[HALF + 1][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    h[0][i] = half ? h1[i] : h0[i];
#pragma unroll
                for (int u = 0; u < HALF; ++u) {
                    const int at = half * HALF + u;
                    const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[at * (CH / 2) + pair];
                    f2 a[4];
                    decays(a, my.A2, tok.x);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        h[u + 1][i] = h[u][i];
                    advance(h[u + 1], a, tok.y, reinterpret_cast<const float4*>(s_B)[at * LANES + sub]);
                    if (want_z) {
                        const float4 c4 = reinterpret_cast<const float4*>(s_C)[at * LANES + sub];
                        const float c[4] = {c4.x, c4.y, c4.z, c4.w};
                        float y0 = 0.f, y1 = 0.f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float a0, a1;
                            unpack2(h[u + 1][i], a0, a1);
                            y0 = fmaf(a0, c[i], y0), y1 = fmaf(a1, c[i], y1);
                        }
                        put_aside(s_y + u * (CH / 2 * LANES) + tid, y0, y1);
                    }
                }
#pragma unroll
                for (int u = HALF - 1; u >= 0; --u) {
                    const int at = half * HALF + u;
                    const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[at * (CH / 2) + pair];
                    const float2 g = s_g[at * (CH / 2) + pair];
                    const float4 b4 = reinterpret_cast<const float4*>(s_B)[at * LANES + sub], c4 = reinterpret_cast<const float4*>(s_C)[at * LANES + sub];
                    const float b[4] = {b4.x, b4.y, b4.z, b4.w}, c[4] = {c4.x, c4.y, c4.z, c4.w};
                    f2 a[4], through = 0;
                    decays(a, my.A2, tok.x);
                    float in0, in1, bc[8], qB0 = 0.f, qB1 = 0.f;
                    unpack2(tok.y, in0, in1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float q0, q1, s0, s1;                        // q_t, h_t
                        unpack2(r[i], q0, q1);
                        q0 = fmaf(g.x, c[i], q0), q1 = fmaf(g.y, c[i], q1);
                        const f2 co = pack2(q0, q1);
                        unpack2(h[u + 1][i], s0, s1);
                        bc[i] = fmaf(q1, in1, q0 * in0);
                        bc[4 + i] = fmaf(s1, g.y, s0 * g.x);
                        qB0 = fmaf(q0, b[i], qB0), qB1 = fmaf(q1, b[i], qB1);
                        r[i] = mul2(a[i], co);
                        const f2 qah = mul2(r[i], h[u][i]);
                        dA[i] = fma2(tok.x, qah, dA[i]);
                        through = fma2(my.A2[i], qah, through);
                    }
                    float th0, th1;
                    unpack2(through, th0, th1);
                    put_aside(s_q + u * (CH / 2 * LANES) + tid, qB0, qB1, th0, th1);
                    group_sums<8, 32 / LANES, LANES>(bc, lane);
                    constexpr int W = 32 / LANES, kept = W >= 8 ? 1 : 8 / W;
                    const int j = lane / LANES, first = first_value<8, W>(j);
                    if (W <= 8 || j < 8)
#pragma unroll
                        for (int i = 0; i < kept; ++i) {
                            const int v = first + i;
                            put_aside(s_BC + ((warp * HALF + u) * 2 + v / 4) * NP + n0 + v % 4, bc[i]);
                        }
                    asm volatile("" ::: "memory");                   // keeps the loads of a token with its products
                }
                __syncthreads();
                // shares of dB and dC of this block's channels
                if (p.part_BC) {
                    const long long at0 = slot * kPiece + half * HALF, rows = p.runs * kRun * kPiece;
                    float* to = p.part_BC + (((long long)block * rows + at0) * p.f.groups + group) * 2 * NP;
                    for (int at = tid; at < HALF * 2 * NP; at += kGradThreads) {
                        const int u = at / (2 * NP), v = at % (2 * NP);
                        float s = 0.f;
#pragma unroll
                        for (int w = 0; w < WARPS; ++w)
                            s += s_BC[(w * HALF + u) * 2 * NP + v];
                        to[(long long)u * p.f.groups * 2 * NP + v] = s;
                    }
                }
                // gradients of this thread's tokens
#pragma unroll
                for (int e = 0; e < L::PASSES; ++e) {
                    const int u = e * L::ROWS + tile.lr;
                    if (u / HALF != half || u >= left || !tile.mine)
                        continue;
                    const int at = (u % HALF * (CH / 2) + tile.lc / 2) * LANES;
                    float4 s = s_q[at];
#pragma unroll
                    for (int i = 1; i < LANES; ++i) {
                        const float4 m = s_q[at + i];
                        s.x += m.x, s.y += m.y, s.z += m.z, s.w += m.w;
                    }
                    float2 y = make_float2(0.f, 0.f);
                    if (want_z) {
                        y = s_y[at];
#pragma unroll
                        for (int i = 1; i < LANES; ++i) {
                            const float2 m = s_y[at + i];
                            y.x += m.x, y.y += m.y;
                        }
                    }
                    const float* steps = reinterpret_cast<const float*>(s_tok + u * (CH / 2) + tile.lc / 2) + tile.lc % 2;
                    const float* gs = reinterpret_cast<const float*>(s_g + u * (CH / 2) + tile.lc / 2) + tile.lc % 2;
                    Vec<T, V> dx, ddelta, dz;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const bool odd = V == 2 ? v : tile.lc % 2;
                        const float qB = odd ? s.y : s.x, th = odd ? s.w : s.z, step = steps[v], g = gs[v], x = to_f(tile.x[e].v[v]);
                        dx.v[v] = from_f<T>(fmaf(step, qB, skip[v] * g));
                        float d = fmaf(x, qB, th * (1.f / kLog2e));
                        if (p.f.softplus) {
                            // the logistic function of what the softplus was given, 1 - exp(-D); a series where that cancels
                            const float small = step * fmaf(step, fmaf(step, fmaf(step, -1.f / 24, 1.f / 6), -0.5f), 1.f);
                            d *= step < 0.06f ? small : 1.f - ex2(step * -kLog2e);
                        }
                        ddelta.v[v] = from_f<T>(d);
                        if (want_z) {
                            const float z = to_f(tile.z[e].v[v]);
                            dz.v[v] = from_f<T>(to_f(tile.dy[e].v[v]) * fmaf(skip[v], x, odd ? y.y : y.x) * silu_slope(z));
                        }
                        sum_D[v] = fmaf(g, x, sum_D[v]);
                        sum_bias[v] += d;
                    }
                    const long long to = row + u;
                    if (p.dx.ptr)
                        *reinterpret_cast<Vec<T, V>*>(row_ptr<T>(p.dx, q.seq, to) + tile.chan) = dx;
                    if (p.ddelta.ptr)
                        *reinterpret_cast<Vec<T, V>*>(row_ptr<T>(p.ddelta, q.seq, to) + tile.chan) = ddelta;
                    if (want_z)
                        *reinterpret_cast<Vec<T, V>*>(row_ptr<T>(p.dz, q.seq, to) + tile.chan) = dz;
                }
                __syncthreads();
            }
        }
    }
    if (p.part_A)
        my.set(p.part_A + (long long)blockIdx.x * states, dA, p.f.vec4);
    if (p.part_D) {
        // a channel's sums lie with the ROWS threads that load it
        float* sums = reinterpret_cast<float*>(s_q);                 // [2][ROWS][CH]
        if (tile.mine)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                sums[tile.lr * CH + tile.lc + v] = sum_D[v];
                sums[(L::ROWS + tile.lr) * CH + tile.lc + v] = sum_bias[v];
            }
        __syncthreads();
        constexpr int held = L::ROWS < kPiece ? L::ROWS : kPiece;
        for (int c = tid; c < 2 * CH; c += kGradThreads) {
            const int kind = c / CH, ch = c % CH;
            if (c0 + ch >= per_group)
                continue;
            float s = 0.f;
            for (int i = 0; i < held; ++i)
                s += sums[(kind * L::ROWS + i) * CH + ch];
            p.part_D[((long long)blockIdx.x * 2 + kind) * p.f.d + group * per_group + c0 + ch] = s;
        }
    }
}

// Sums over the runs, dA first, then dD and ddelta_bias: out[i] = sum_r part[r][i], 32 of them to a block.  Runs without a
// sequence were not written.
static __global__ void __launch_bounds__(256) grad_sum_kernel(const GradDev p)
{
    wait_for_previous();
    __shared__ float sum[8][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const long long states = (long long)p.f.d * p.f.n, a_blocks = p.dA ? (states + 31) / 32 : 0, d_blocks = (p.f.d + 31) / 32;
    const long long b = blockIdx.x - a_blocks;
    const bool of_A = b < 0;
    const int kind = of_A ? 0 : static_cast<int>(b / d_blocks);      // 0: dD, 1: ddelta_bias
    const long long i = (of_A ? blockIdx.x : b % d_blocks) * 32 + lane, size = of_A ? states : p.f.d, stride = of_A ? states : 2ll * p.f.d;
    const float* part = of_A ? p.part_A : p.part_D + kind * p.f.d;
    float* out = of_A ? p.dA : kind ? p.ddelta_bias : p.dD;
    const long long runs = p.f.piece_map ? p.f.seq_first[p.f.seqs.batch] : p.runs;
    float s = 0.f;
    if (i < size)
        for (long long r = warp; r < runs; r += 8)
            s += part[r * stride + i];
    sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && i < size && out) {
        for (int k = 1; k < 8; ++k)
            s += sum[k][lane];
        out[i] = s;
    }
}

// dB and dC of every token: the channel blocks of its group added up.
template <typename T> __global__ void __launch_bounds__(256) grad_rows_kernel(const GradDev p, int NP)
{
    wait_for_previous();
    Piece q;
    if (!find_piece(p.f, blockIdx.x, q))
        return;
    const long long rows = p.runs * kRun * kPiece, per_row = (long long)p.f.groups * 2 * NP;
    const int tokens = static_cast<int>(q.t1 - q.t0);
    for (long long at = (long long)blockIdx.y * 256 + threadIdx.x; at < tokens * per_row; at += (long long)gridDim.y * 256) {
        const long long u = at / per_row;
        const int v = static_cast<int>(at % per_row), group = v / (2 * NP), kind = v / NP % 2, k = v % NP;
        const Rows& out = kind ? p.dC : p.dB;
        if (k >= p.f.n || !out.ptr)
            continue;
        const float* from = p.part_BC + ((long long)blockIdx.x * kRun * kPiece + u) * per_row + v;
        float s = 0.f;
        for (int b = 0; b < p.f.chan_blocks; ++b)
            s += from[b * rows * per_row];
        row_ptr<T>(out, q.seq, q.row0 + q.t0 + u)[group * p.f.n + k] = from_f<T>(s);
    }
}

} // namespace sscan
} // namespace ttc
