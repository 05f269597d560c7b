// Selective state space scan: h_t = exp(D_t A) h_{t-1} + D_t x_t B_t, y_t = (C_t . h_t + D x_t) silu(z_t), diagonal A.
//
// A channel's n states are spread over LANES neighbouring lanes, four to a lane; a lane holds them for two neighbouring
// channels, as packed pairs (even channel, odd channel).  A block owns 256 / LANES channels of one group and walks over the
// tokens in tiles.
// Four of its warps run the recurrence; eight load the rows, compute the step size (bias, softplus) and D_t x_t of
// every token and channel once, leave them in shared memory with B and C in float32, and take the lanes' shares of C . h
// from there to the output rows.  Both work at the same time, on tiles next to one another, with one barrier for each tile.
// Padding tokens have D_t = 0 (a = 1, nothing added) and padding states A = B = C = 0, so neither needs a test.
// Per state and token: one exponential, four multiply-adds and six bytes from shared memory.  The special-function unit (16
// exponentials per clock and SM) bounds it, with shared memory close behind: a 16-byte load occupies the return path for four
// clocks, broadcast or not, and with one channel to a lane (twelve bytes) that path was the bound.
//
// 4 sequences of 2048 tokens, 4096 channels, 16 states, bfloat16: 250 us, 2.15e12 states a second, the unit at 60 % (137 us would
// be all of it with what softplus and gate ask for), issue slots 59 %; 256 blocks on 148 SMs leave some with one.  On the way:
// every warp loading and stepping, one channel to a lane 338 us, two channels 532 (too few warps), warps with roles 324 with
// four for the rows and 283 with eight, loads without branches 256, tiles of 32 tokens 250 (at 16 states; 8 and 16 where
// other widths are fastest).
//
// Few channels: the tokens are cut into pieces.  A first pass (LOCAL: recurrence without outputs) finds what each piece adds to
// the state, from zero, and the sum of its steps; the second takes the state in front of its piece from those, since a
// piece's decay is exp(A sum D_t).  16381 tokens, 1024 channels, 16 states: 84 + 115 us, twice the exponentials.
#pragma once

#include <type_traits>

#include "pieces.cuh"

namespace ttc {
namespace sscan {

using namespace blk;

constexpr int kStepThreads = 128;
constexpr int kStateThreads = 128, kRowThreads = 256, kThreads = kStateThreads + kRowThreads;   // of a block: run the recurrence; load and store
// what a block of the scan holds
constexpr int channels_of(int lanes) { return 2 * kStateThreads / lanes; }

struct ScanDev {
    Seqs seqs;
    int d, n, groups, softplus;
    int chan_blocks;              // blocks of channels per group
    Rows x, delta, B, C, z, y;
    const float *A, *D, *delta_bias, *state;
    float* state_out;
    // the horizon cut into pieces of `piece` tokens (0: every sequence is one piece)
    long long piece, pieces_per_seq;
    const int2* piece_map;        // packed: {sequence, first token} of every piece, sequence -1: none
    const int* seq_first;         // packed: first piece of every sequence, [batch + 1]
    int vec4;                     // rows of state and A can be read by four floats
    float *local, *local_step;    // [pieces][d][n] and [pieces][d]: what a piece adds to a state, and its sum of D_t
};

// A log2(e).  Minus infinity becomes the lowest number: times a step of 0 (of a padding token, or a softplus that underflows) it has to be 0.
__device__ __forceinline__ float exponent(float A)
{
    const float e = A * kLog2e;
    return e < -3.4e38f ? -3.4e38f : e;
}

struct Piece {
    long long seq, t0, t1, row0, len;
    long long first, last;        // pieces of the same sequence
};

__device__ __forceinline__ bool find_piece(const ScanDev& p, long long i, Piece& q)
{
    if (p.piece_map) {
        const int2 m = p.piece_map[i];
        if (m.x < 0)
            return false;
        q.seq = m.x;
        q.t0 = m.y;
        q.first = p.seq_first[q.seq];
        q.last = p.seq_first[q.seq + 1] - 1;
    } else {
        q.seq = i / p.pieces_per_seq;
        q.first = q.seq * p.pieces_per_seq;
        q.last = q.first + p.pieces_per_seq - 1;
        q.t0 = (i - q.first) * p.piece;
    }
    const Span s = span_of(p.seqs, q.seq);
    q.row0 = s.row0;
    q.len = s.len;
    q.t1 = p.piece && q.t0 + p.piece < s.len ? q.t0 + p.piece : s.len;
    return true;
}

// Rows of a tile in the order in which a block's threads load them: V neighbouring columns to a thread, ROWS rows to a pass.
template <int WIDTH, int TB, int V> struct Lay {
    static constexpr int COLS = WIDTH / V, ROWS = kRowThreads / COLS, PASSES = (TB + ROWS - 1) / ROWS;
    static_assert(WIDTH % V == 0 && kRowThreads % COLS == 0, "");
};

template <int LANES> struct Shape {
    static constexpr int CH = channels_of(LANES);
    static constexpr int NP = LANES * 4;                // padded states
    static constexpr int TB = LANES == 2 ? 8 : LANES == 4 ? 32 : 16;
    static constexpr int TOK = TB * CH * 2, BC = TB * NP, Y = TB * CH * LANES;      // floats of a buffer
    static constexpr size_t smem(bool local) { return 2 * sizeof(float) * (TOK + BC * (local ? 1 : 2) + (local ? 0 : Y)); }
};

// A row operand as a thread walks over it: its own columns, ROWS rows further at each pass.
template <typename T, int V, int PASSES> struct Walk {
    const T* at;
    long long pass, tile;
    __device__ __forceinline__ void start(const Rows& r, long long seq, long long row, int col, int rows_per_pass, int tile_rows)
    {
        at = row_ptr<const T>(r, seq, row) + col;
        pass = rows_per_pass * r.ts;
        tile = tile_rows * r.ts;
    }
    // rows from `row` on, ROWS apart, as long as they are below `rows`; the rest reads as zero
    template <int ROWS> __device__ __forceinline__ void load(Vec<T, V> (&raw)[PASSES], bool mine, int row, int rows)
    {
        const T* from = at;
#pragma unroll
        for (int e = 0; e < PASSES; ++e, from += pass)
            raw[e] = load_if(reinterpret_cast<const Vec<T, V>*>(from), mine && row + e * ROWS < rows);
        at += tile;
    }
};

template <int V> __device__ __forceinline__ void put(float* to, const float (&v)[V])
{
    if constexpr (V == 2) {
        *reinterpret_cast<float2*>(to) = make_float2(v[0], v[1]);
    } else {
        to[0] = v[0];
    }
}

__device__ __forceinline__ void meet() { asm volatile("barrier.sync 0, %0;" :: "n"(kThreads) : "memory"); }

// The recurrence: four states of two channels.
template <int LANES, bool LOCAL>
__device__ __forceinline__ void run_states(const ScanDev& p, const Piece& q, int group, int per_group, int c0, const float4* s_tok, const float* s_B,
                                           const float* s_C, float2* s_y, int tiles)
{
    using S = Shape<LANES>;
    constexpr int CH = S::CH, TB = S::TB;
    const int tid = threadIdx.x, sub = tid % LANES, pair = tid / LANES, n0 = sub * 4;
    f2 A2[4], h2[4], total = 0;                                      // pairs of channels
    {
        float a[2][4], h[2][4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const bool have = c0 + 2 * pair + c < per_group;
            const long long my = group * per_group + c0 + 2 * pair + c;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool ok = have && n0 + i < p.n;
                a[c][i] = ok ? exponent(p.A[my * p.n + n0 + i]) : 0.f;
                h[c][i] = !LOCAL && !p.piece && ok && p.state ? p.state[(q.seq * p.d + my) * p.n + n0 + i] : 0.f;
            }
            // (state itself may be overwritten already by the last piece)
            if (!LOCAL && p.piece && have) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n0 + i < p.n)
                        h[c][i] = p.local[(q.last * p.d + my) * p.n + n0 + i];
                for (long long k = q.first; k < (long long)blockIdx.x; ++k) {
                    const float step = p.local_step[k * p.d + my];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n0 + i < p.n)
                            h[c][i] = fmaf(ex2(a[c][i] * step), h[c][i], p.local[(k * p.d + my) * p.n + n0 + i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            A2[i] = pack2(a[0][i], a[1][i]);
            h2[i] = pack2(h[0][i], h[1][i]);
        }
    }
    meet();
    for (int tile = 0; tile < tiles; ++tile) {
        const ulonglong2* tok = reinterpret_cast<const ulonglong2*>(s_tok) + (tile & 1) * (S::TOK / 4) + pair;
        const float4* Bs = reinterpret_cast<const float4*>(s_B) + (tile & 1) * (S::BC / 4) + sub;
        const float4* Cs = reinterpret_cast<const float4*>(s_C) + (tile & 1) * (S::BC / 4) + sub;
        float2* ys = s_y + (tile & 1) * (S::Y / 2) + tid;
        // The exponentials of the next token are issued before the products of this one, so that the special-function unit
        // does not wait for them.
        f2 next[4];
        ulonglong2 tok_next;
        auto decays = [&](int u) {
            tok_next = tok[u * (CH / 2)];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float e0, e1;
                unpack2(fma2(A2[i], tok_next.x, pack2(kExBias, kExBias)), e0, e1);
                next[i] = pack2(ex2(e0), ex2(e1));
            }
            if (LOCAL)
                total = add2(total, tok_next.x);
        };
        decays(0);
#pragma unroll 8
        for (int u = 0; u < TB; ++u) {
            f2 a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[i] = next[i];
            float in0, in1, y0, y1;
            unpack2(tok_next.y, in0, in1);
            if (u + 1 < TB)
                decays(u + 1);
            const float4 b4 = Bs[u * LANES];
            const float b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                h2[i] = fma2(a[i], h2[i], pack2(in0 * b[i], in1 * b[i]));
            if (!LOCAL) {
                const float4 c4 = Cs[u * LANES];
                const float c[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float h0, h1;
                    unpack2(h2[i], h0, h1);
                    y0 = i ? fmaf(h0, c[i], y0) : h0 * c[i];
                    y1 = i ? fmaf(h1, c[i], y1) : h1 * c[i];
                }
                put_aside(ys + u * (CH / 2 * LANES), y0, y1);
            }
        }
        meet();
    }
    float h[2][4], steps[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        unpack2(h2[i], h[0][i], h[1][i]);
    unpack2(total, steps[0], steps[1]);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        if (c0 + 2 * pair + c >= per_group)
            continue;
        const long long my = group * per_group + c0 + 2 * pair + c;
        float* to = LOCAL ? p.local + ((long long)blockIdx.x * p.d + my) * p.n : p.state_out && q.t1 == q.len ? p.state_out + (q.seq * p.d + my) * p.n : nullptr;
        if (to)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < p.n)
                    to[n0 + i] = h[c][i];
        if (LOCAL && sub == 0)
            p.local_step[(long long)blockIdx.x * p.d + my] = steps[c];
    }
}

// The rows: tile i + 1 is staged and the output of tile i - 1 is written while the recurrence runs over tile i; the loads of
// tile i + 2 (of z: i) are under way meanwhile.
template <typename T, int LANES, bool LOCAL, int V>
__device__ __forceinline__ void run_rows(const ScanDev& p, const Piece& q, int group, int per_group, int c0, float4* s_tok, float* s_B, float* s_C,
                                         const float2* s_y, int tiles)
{
    using S = Shape<LANES>;
    constexpr int CH = S::CH, NP = S::NP, TB = S::TB;
    using LT = Lay<CH, TB, V>;                                       // token rows
    using LB = Lay<NP, TB, V>;                                       // rows of B and C
    constexpr int PASSES = LT::PASSES;
    const int tid = threadIdx.x - kStateThreads;
    // first of the channels, and first row of a tile, that this thread loads and stores; the same for B and C
    const int lc = tid % LT::COLS * V, lr = tid / LT::COLS;
    const int chan = group * per_group + c0 + lc;
    const bool have_l = c0 + lc < per_group && lr < TB;
    const int bc = tid % LB::COLS * V, br = tid / LB::COLS;
    const bool have_b = bc < p.n && br < TB;
    const bool gated = !LOCAL && p.z.ptr;
    float bias[V], skip[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = p.delta_bias && have_l ? p.delta_bias[chan + v] : 0.f;
        skip[v] = !LOCAL && p.D && have_l ? p.D[chan + v] : 0.f;
    }
    const int len = static_cast<int>(q.t1 - q.t0);
    const long long row = q.row0 + q.t0;
    Walk<T, V, PASSES> x, delta, z;
    Walk<T, V, LB::PASSES> B, C;
    x.start(p.x, q.seq, row + lr, chan, LT::ROWS, TB);
    delta.start(p.delta, q.seq, row + lr, chan, LT::ROWS, TB);
    z.start(p.z, q.seq, row + lr, chan, LT::ROWS, TB);
    B.start(p.B, q.seq, row + br, group * p.n + bc, LB::ROWS, TB);
    C.start(p.C, q.seq, row + br, group * p.n + bc, LB::ROWS, TB);
    T* y = row_ptr<T>(p.y, q.seq, row + lr) + chan;
    const long long y_pass = LT::ROWS * p.y.ts, y_tile = TB * p.y.ts;

    struct Raw {
        Vec<T, V> x[PASSES], delta[PASSES], z[PASSES], B[LB::PASSES], C[LB::PASSES];
    };
    auto load_rows = [&](Raw& r, int tile) {
        const int left = len - tile * TB;
        x.template load<LT::ROWS>(r.x, have_l, lr, left);
        delta.template load<LT::ROWS>(r.delta, have_l, lr, left);
        B.template load<LB::ROWS>(r.B, have_b, br, left);
        if (!LOCAL)
            C.template load<LB::ROWS>(r.C, have_b, br, left);
    };
    auto load_gate = [&](Raw& r, int tile) { z.template load<LT::ROWS>(r.z, have_l && gated, lr, len - tile * TB); };
    auto tokens = [&](auto full, const Raw& r, int left, float4* to) {
        constexpr bool FULL = decltype(full)::value;
#pragma unroll
        for (int e = 0; e < PASSES; ++e) {
            const int u = e * LT::ROWS + lr;
            const bool none = !FULL && u >= left;                    // padding: nothing decays, nothing is added
            float4* at = to + u * (CH / 2) + lc / 2;
            if constexpr (V == 2) {
                f2 step = add2(pack2(to_f(r.delta[e].v[0]), to_f(r.delta[e].v[1])), pack2(bias[0], bias[1]));
                if (p.softplus)
                    step = softplus2(step);
                const f2 in = mul2(step, pack2(to_f(r.x[e].v[0]), to_f(r.x[e].v[1])));
                *reinterpret_cast<ulonglong2*>(at) = none ? make_ulonglong2(0, 0) : make_ulonglong2(step, in);
            } else {
                float step = to_f(r.delta[e].v[0]) + bias[0];
                if (p.softplus)
                    step = softplus(step);
                reinterpret_cast<float*>(at)[lc % 2] = none ? 0.f : step;
                reinterpret_cast<float*>(at)[2 + lc % 2] = none ? 0.f : step * to_f(r.x[e].v[0]);
            }
        }
    };
    auto stage = [&](const Raw& r, int tile) {
        const int left = len - tile * TB;
        if (LT::ROWS <= TB || lr < TB) {
            float4* to = s_tok + (tile & 1) * (S::TOK / 4);
            if (left >= TB)
                tokens(std::true_type(), r, left, to);
            else
                tokens(std::false_type(), r, left, to);
        }
        if (LB::ROWS <= TB || br < TB) {
#pragma unroll
            for (int e = 0; e < LB::PASSES; ++e) {
                const int at = (tile & 1) * S::BC + (e * LB::ROWS + br) * NP + bc;
                float b[V], c[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    b[v] = to_f(r.B[e].v[v]), c[v] = LOCAL ? 0.f : to_f(r.C[e].v[v]);
                put<V>(s_B + at, b);
                if (!LOCAL)
                    put<V>(s_C + at, c);
            }
        }
    };
    Vec<T, V> x0[PASSES], x1[PASSES];                                // x of the tiles whose output is still to be written
    auto keep = [&](const Raw& r) {
        if (!LOCAL)
#pragma unroll
            for (int e = 0; e < PASSES; ++e)
                x0[e] = x1[e], x1[e] = r.x[e];
    };
    auto give = [&](const Raw& of, int tile) {
        const int left = len - tile * TB;
        const float2* shares = s_y + (tile & 1) * (S::Y / 2);
        const int swap = (lc / 2 ^ lc / 8) & 1;                      // neighbours begin with different banks
        T* to = y;
#pragma unroll
        for (int e = 0; e < PASSES; ++e, to += y_pass) {
            const int u = e * LT::ROWS + lr;
            if (have_l && u < left) {
                Vec<T, V> out;
                f2 s2 = 0;
                const ulonglong2* from = reinterpret_cast<const ulonglong2*>(shares + (u * (CH / 2) + lc / 2) * LANES);
#pragma unroll
                for (int k = 0; k < LANES / 2; ++k) {
                    const ulonglong2 two = from[LANES > 2 ? k ^ swap : 0];
                    s2 = k ? add2(s2, add2(two.x, two.y)) : add2(two.x, two.y);
                }
                float r0, r1;
                if constexpr (V == 2) {
                    s2 = fma2(pack2(skip[0], skip[1]), pack2(to_f(x0[e].v[0]), to_f(x0[e].v[1])), s2);
                    if (gated)
                        s2 = mul2(s2, silu2(pack2(to_f(of.z[e].v[0]), to_f(of.z[e].v[1]))));
                    unpack2(s2, r0, r1);
                    out.v[0] = from_f<T>(r0), out.v[1] = from_f<T>(r1);
                } else {
                    unpack2(s2, r0, r1);
                    float r = fmaf(skip[0], to_f(x0[e].v[0]), lc % 2 ? r1 : r0);
                    if (gated)
                        r *= silu(to_f(of.z[e].v[0]));
                    out.v[0] = from_f<T>(r);
                }
                *reinterpret_cast<Vec<T, V>*>(to) = out;
            }
        }
        y += y_tile;
    };
    Raw raw;
    if (tiles) {
        load_rows(raw, 0);
        stage(raw, 0);
        keep(raw);
        load_rows(raw, 1);
        load_gate(raw, 0);
    }
    meet();
    for (int tile = 0; tile < tiles; ++tile) {
        if (!LOCAL && tile > 0)
            give(raw, tile - 1);
        if (tile + 1 < tiles)
            stage(raw, tile + 1);
        keep(raw);
        // Issued when nothing is left to wait for: a warp that waits for older loads waits for younger ones with them.
        load_rows(raw, tile + 2);
        if (tile > 0)
            load_gate(raw, tile);
        meet();
    }
    if (!LOCAL && tiles)
        give(raw, tiles - 1);
}

// LOCAL: what a piece adds to the state that enters it (from zero), and the sum of its step sizes; no output rows.
template <typename T, int LANES, bool LOCAL, int V>
__global__ void __launch_bounds__(kThreads, 2) scan_kernel(const ScanDev p)
{
    using S = Shape<LANES>;
    extern __shared__ float4 smem[];
    float4* s_tok = smem;                                            // [2][TB][CH / 2]: D_t and D_t x_t of two channels
    float* s_B = reinterpret_cast<float*>(s_tok) + 2 * S::TOK;       // [2][TB][NP]
    float* s_C = s_B + 2 * S::BC;
    float2* s_y = reinterpret_cast<float2*>(s_C + 2 * S::BC);        // [2][TB][CH / 2][LANES]: each lane's share of C . h

    Piece q;
    if (!find_piece(p, blockIdx.x, q))
        return;
    const int group = blockIdx.y / p.chan_blocks, per_group = p.d / p.groups;
    const int c0 = (blockIdx.y % p.chan_blocks) * S::CH;             // first channel, within the group
    if (LOCAL && q.last == blockIdx.x) {
        // The last piece's own share is not needed: its place keeps the state in front of the sequence, which the pass that
        // follows may overwrite.
        const long long first = group * per_group + c0, count = (long long)min(S::CH, per_group - c0) * p.n;
        for (long long i = threadIdx.x; i < count; i += kThreads)
            p.local[((long long)blockIdx.x * p.d + first) * p.n + i] = p.state ? p.state[(q.seq * p.d + first) * p.n + i] : 0.f;
        return;
    }
    const int tiles = static_cast<int>((q.t1 - q.t0 + S::TB - 1) / S::TB);
    if (threadIdx.x < kStateThreads)
        run_states<LANES, LOCAL>(p, q, group, per_group, c0, s_tok, s_B, s_C, s_y, tiles);
    else
        run_rows<T, LANES, LOCAL, V>(p, q, group, per_group, c0, s_tok, s_B, s_C, s_y, tiles);
}

// One token of each sequence: the state is read and written once, which is what bounds it; for few sequences the latency of
// one round of loads (16 sequences, 4096 channels, 16 states: 4.3 us for 8.9 MB).
template <typename T, int LANES>
__global__ void __launch_bounds__(kStepThreads, 12) scan_step_kernel(const ScanDev p)
{
    wait_for_previous();
    constexpr int CH = kStepThreads / LANES;
    const int tid = threadIdx.x, sub = tid % LANES, ch = tid / LANES;
    const long long b = blockIdx.x;
    const int c = blockIdx.y * CH + ch;
    const bool have = c < p.d;
    const int n0 = sub * 4;
    float y[1] = {0.f};
    float x = 0.f, gate = 1.f, skip = 0.f;
    if (have) {
        const int first = c / (p.d / p.groups) * p.n + n0, count = min(4, p.n - n0);
        float* st = p.state_out + (b * p.d + c) * p.n + n0;
        const float* A = p.A + (long long)c * p.n + n0;
        const T* B = row_ptr<const T>(p.B, b, 0) + first;
        const T* C = row_ptr<const T>(p.C, b, 0) + first;
        float h[4] = {}, a[4] = {}, bb[4] = {}, cc[4] = {};
        x = to_f(row_ptr<const T>(p.x, b, 0)[c]);
        float step = to_f(row_ptr<const T>(p.delta, b, 0)[c]) + (p.delta_bias ? p.delta_bias[c] : 0.f);
        if (p.vec4) {
            if (count > 0) {
                const float4 v = *reinterpret_cast<const float4*>(st), w = *reinterpret_cast<const float4*>(A);
                h[0] = v.x, h[1] = v.y, h[2] = v.z, h[3] = v.w;
                a[0] = w.x, a[1] = w.y, a[2] = w.z, a[3] = w.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count)
                    h[i] = st[i], a[i] = A[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count)
                bb[i] = to_f(B[i]), cc[i] = to_f(C[i]);
        if (sub == 0) {
            skip = p.D ? p.D[c] : 0.f;
            if (p.z.ptr)
                gate = silu(to_f(row_ptr<const T>(p.z, b, 0)[c]));
        }
        if (p.softplus)
            step = softplus(step);
        const float v = step * x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = fmaf(ex2(fmaf(step, exponent(a[i]), kExBias)), h[i], v * bb[i]);
            y[0] = fmaf(h[i], cc[i], y[0]);
        }
        if (p.vec4) {
            if (count > 0)
                *reinterpret_cast<float4*>(st) = make_float4(h[0], h[1], h[2], h[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count)
                    st[i] = h[i];
        }
    }
    group_sums<1, LANES, 1>(y, tid);
    if (have && sub == 0)
        row_ptr<T>(p.y, b, 0)[c] = from_f<T>(fmaf(skip, x, y[0]) * gate);
}

} // namespace sscan
} // namespace ttc
