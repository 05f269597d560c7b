// Selective state space scan: h_t = exp(D_t A) h_{t-1} + D_t x_t B_t, y_t = (C_t . h_t + D x_t) silu(z_t), diagonal A.
//
// A channel's n states are spread over LANES neighbouring lanes, four to a lane (two packed pairs), so a block of 128
// threads owns 128 / LANES channels of one group and walks over the tokens.  Tiles of tokens are staged in shared memory:
// the step size (after bias and softplus) and D_t x_t of every token and channel, computed once, doubled up as operands of
// packed arithmetic, and B, C of the group in float32; the next tile's rows are loaded while this one is computed.
// Padding tokens have D_t = 0 (a = 1, nothing added) and padding states A = B = C = 0, so neither needs a test.
// Per state and token: one exponential and four multiply-adds; the special-function unit (16 exponentials per clock and
// SM) bounds it, before memory (four elements per channel and token) and issue slots.
#pragma once

#include "block_common.cuh"

namespace ttc {
namespace sscan {

using namespace blk;

constexpr int kThreads = 128;
constexpr float kLog2e = 1.4426950408889634f;

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

template <int LANES> struct Shape {
    static constexpr int CH = kThreads / LANES;         // channels of a block
    static constexpr int NP = LANES * 4;                // padded states
    static constexpr int TB = LANES == 1 ? 16 : LANES <= 8 ? 32 : 16;
    static constexpr int EPT = (TB * CH + kThreads - 1) / kThreads;
    static constexpr int BPT = (TB * NP + kThreads - 1) / kThreads;
    static constexpr size_t smem(bool local) { return sizeof(float) * (TB * CH * 4 + TB * NP * (local ? 1 : 2) + (local ? 0 : TB * CH)); }
};

// LOCAL: what a piece adds to the state that enters it (from zero), and the sum of its step sizes; no output rows.
template <typename T, int LANES, bool LOCAL>
__global__ void __launch_bounds__(kThreads) scan_kernel(const ScanDev p)
{
    using S = Shape<LANES>;
    constexpr int CH = S::CH, NP = S::NP, TB = S::TB, EPT = S::EPT, BPT = S::BPT;
    extern __shared__ float4 smem[];
    float4* s_tok = smem;                                            // [TB][CH]: D_t, D_t, D_t x_t, D_t x_t
    float* s_B = reinterpret_cast<float*>(s_tok + TB * CH);          // [TB][NP]
    float* s_C = s_B + TB * NP;
    float* s_y = s_C + TB * NP;                                      // [TB][CH]

    Piece q;
    if (!find_piece(p, blockIdx.x, q))
        return;
    const int tid = threadIdx.x, sub = tid % LANES, ch = tid / LANES;
    const int group = blockIdx.y / p.chan_blocks, per_group = p.d / p.groups;
    const int c0 = (blockIdx.y % p.chan_blocks) * CH;                // first channel, within the group
    const int my = group * per_group + c0 + ch;                      // this thread's channel
    const bool have = c0 + ch < per_group;
    const int n0 = sub * 4;
    // channel and first token of a tile that this thread loads and stores: token e * (kThreads / CH) + lt
    const int lc = tid % CH, lt = tid / CH;
    const int chan = group * per_group + c0 + lc;
    const bool have_l = c0 + lc < per_group;

    f2 A2[2], h2[2];
    float h[4];
    {
        float a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool ok = have && n0 + i < p.n;
            a[i] = ok ? p.A[(long long)my * p.n + n0 + i] * kLog2e : 0.f;
            h[i] = 0.f;
            if (LOCAL ? q.last == blockIdx.x : q.t0 == 0) {
                if (ok && p.state)
                    h[i] = p.state[(q.seq * p.d + my) * p.n + n0 + i];
            }
        }
        if (LOCAL) {
            // The last piece's own share is not needed: its place keeps the state in front of the sequence, which the
            // pass that follows may overwrite.
            if (q.last == blockIdx.x) {
                for (int i = 0; i < 4; ++i)
                    if (have && n0 + i < p.n)
                        p.local[((long long)blockIdx.x * p.d + my) * p.n + n0 + i] = h[i];
                return;
            }
        } else if (q.t0 > 0) {
            for (int i = 0; i < 4; ++i)
                if (have && n0 + i < p.n)
                    h[i] = p.local[(q.last * p.d + my) * p.n + n0 + i];
            for (long long k = q.first; k < (long long)blockIdx.x; ++k) {
                const float step = have ? p.local_step[k * p.d + my] : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (have && n0 + i < p.n)
                        h[i] = fmaf(ex2(a[i] * step), h[i], p.local[(k * p.d + my) * p.n + n0 + i]);
            }
        }
        A2[0] = pack2(a[0], a[1]), A2[1] = pack2(a[2], a[3]);
        h2[0] = pack2(h[0], h[1]), h2[1] = pack2(h[2], h[3]);
    }
    const float bias = p.delta_bias && have_l ? p.delta_bias[chan] : 0.f;
    const float skip = !LOCAL && p.D && have_l ? p.D[chan] : 0.f;
    const long long seq = q.seq;

    T rx[EPT], rd[EPT], rz[EPT], rB[BPT], rC[BPT];
    auto load = [&](long long t) {
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const long long u = t + e * (kThreads / CH) + lt;
            const bool ok = have_l && u < q.t1 && (TB * CH >= kThreads || lt < TB);
            rx[e] = rd[e] = rz[e] = from_f<T>(0.f);
            if (ok) {
                rx[e] = row_ptr<const T>(p.x, seq, q.row0 + u)[chan];
                rd[e] = row_ptr<const T>(p.delta, seq, q.row0 + u)[chan];
                if (!LOCAL && p.z.ptr)
                    rz[e] = row_ptr<const T>(p.z, seq, q.row0 + u)[chan];
            }
        }
#pragma unroll
        for (int e = 0; e < BPT; ++e) {
            const int at = e * kThreads + tid, u = at / NP, k = at % NP;
            rB[e] = rC[e] = from_f<T>(0.f);
            if (u < TB && t + u < q.t1 && k < p.n) {
                rB[e] = row_ptr<const T>(p.B, seq, q.row0 + t + u)[group * p.n + k];
                if (!LOCAL)
                    rC[e] = row_ptr<const T>(p.C, seq, q.row0 + t + u)[group * p.n + k];
            }
        }
    };
    float xs[EPT], zs[EPT];                                          // of the tile in shared memory
    auto stage = [&](long long t) {
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const int u = e * (kThreads / CH) + lt;
            float step = to_f(rd[e]) + bias;
            if (p.softplus)
                step = softplus(step);
            if (t + u >= q.t1 || !have_l)
                step = 0.f;
            xs[e] = to_f(rx[e]);
            zs[e] = to_f(rz[e]);
            // a padding token adds nothing, whatever step * x would be
            const float v = t + u < q.t1 ? step * xs[e] : 0.f;
            if (u < TB)
                s_tok[u * CH + lc] = make_float4(step, step, v, v);
        }
#pragma unroll
        for (int e = 0; e < BPT; ++e) {
            const int at = e * kThreads + tid;
            if (at < TB * NP) {
                s_B[at] = to_f(rB[e]);
                if (!LOCAL)
                    s_C[at] = to_f(rC[e]);
            }
        }
    };

    float total = 0.f;
    if (q.t0 < q.t1)
        load(q.t0);
    for (long long t = q.t0; t < q.t1; t += TB) {
        stage(t);
        __syncthreads();
        float kx[EPT], kz[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e)
            kx[e] = xs[e], kz[e] = zs[e];
        if (t + TB < q.t1)
            load(t + TB);
#pragma unroll 2
        for (int u = 0; u < TB; u += 4) {
            float part[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[(u + j) * CH + ch];
                const ulonglong2 b = reinterpret_cast<const ulonglong2*>(s_B)[(u + j) * LANES + sub];
                f2 y2 = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float e0, e1;
                    unpack2(mul2(A2[i], tok.x), e0, e1);
                    h2[i] = fma2(pack2(ex2(e0), ex2(e1)), h2[i], mul2(tok.y, i ? b.y : b.x));
                }
                if (LOCAL) {
                    float s, s1;
                    unpack2(tok.x, s, s1);
                    total += s;
                } else {
                    const ulonglong2 c = reinterpret_cast<const ulonglong2*>(s_C)[(u + j) * LANES + sub];
                    y2 = fma2(h2[1], c.y, mul2(h2[0], c.x));
                    part[j] = sum2(y2);
                }
            }
            if (!LOCAL) {
                group_sums<4, LANES, 1>(part, tid);
                constexpr int left = LANES >= 4 ? 1 : 4 / LANES;
                const int first = first_value<4, LANES>(sub);
                if (LANES <= 4 || sub < 4)
#pragma unroll
                    for (int i = 0; i < left; ++i)
                        s_y[(u + first + i) * CH + ch] = part[i];
            }
        }
        __syncthreads();
        if (!LOCAL) {
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                const int u = e * (kThreads / CH) + lt;
                if (u < TB && t + u < q.t1 && have_l) {
                    float y = fmaf(skip, kx[e], s_y[u * CH + lc]);
                    if (p.z.ptr)
                        y *= silu(kz[e]);
                    row_ptr<T>(p.y, seq, q.row0 + t + u)[chan] = from_f<T>(y);
                }
            }
        }
    }
    unpack2(h2[0], h[0], h[1]);
    unpack2(h2[1], h[2], h[3]);
    if (LOCAL) {
        for (int i = 0; i < 4; ++i)
            if (have && n0 + i < p.n)
                p.local[((long long)blockIdx.x * p.d + my) * p.n + n0 + i] = h[i];
        if (have && sub == 0)
            p.local_step[(long long)blockIdx.x * p.d + my] = total;
    } else if (p.state_out && q.t1 == q.len) {
        for (int i = 0; i < 4; ++i)
            if (have && n0 + i < p.n)
                p.state_out[(q.seq * p.d + my) * p.n + n0 + i] = h[i];
    }
}

// Pieces of packed sequences: seq_first [batch + 1], and {sequence, first token} of each; every sequence has at least one
// piece, so that its last state is written.  One block.
static __global__ void __launch_bounds__(1024) piece_map_kernel(Seqs s, long long piece, int at_least, long long bound, int2* map, int* seq_first)
{
    __shared__ int sum[1024];
    __shared__ int base;
    if (threadIdx.x == 0)
        base = 0;
    __syncthreads();
    for (long long b0 = 0; b0 < s.batch; b0 += 1024) {
        const long long b = b0 + threadIdx.x;
        int count = 0;
        if (b < s.batch) {
            const long long c = (span_of(s, b).len + piece - 1) / piece;
            count = static_cast<int>(c < at_least ? at_least : c);
        }
        sum[threadIdx.x] = count;
        __syncthreads();
        for (int o = 1; o < 1024; o *= 2) {
            const int v = threadIdx.x >= o ? sum[threadIdx.x - o] : 0;
            __syncthreads();
            sum[threadIdx.x] += v;
            __syncthreads();
        }
        // offsets that do decrease could ask for more pieces than there is room for: they are cut off
        const long long end = base + (long long)sum[threadIdx.x], first = end - count;
        if (b < s.batch) {
            seq_first[b] = static_cast<int>(first < bound ? first : bound);
            for (int i = 0; i < count && first + i < bound; ++i)
                map[first + i] = make_int2(static_cast<int>(b), static_cast<int>(i * piece));
        }
        __syncthreads();
        if (threadIdx.x == 1023)
            base = static_cast<int>(end < bound ? end : bound);
        __syncthreads();
    }
    if (threadIdx.x == 0)
        seq_first[s.batch] = base;
    for (long long i = base + threadIdx.x; i < bound; i += 1024)
        map[i] = make_int2(-1, 0);
}

// One token of each sequence: the state is read and written once, which is what bounds it.
template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(const ScanDev p)
{
    constexpr int CH = kThreads / LANES;
    const int tid = threadIdx.x, sub = tid % LANES, ch = tid / LANES;
    const long long b = blockIdx.x;
    const int c = blockIdx.y * CH + ch;
    const bool have = c < p.d;
    const int n0 = sub * 4, per_group = p.d / p.groups;
    float y[1] = {0.f};
    float x = 0.f;
    if (have) {
        const int group = c / per_group;
        float* st = p.state_out + (b * p.d + c) * p.n;
        const float* A = p.A + (long long)c * p.n;
        const T* B = row_ptr<const T>(p.B, b, 0) + group * p.n;
        const T* C = row_ptr<const T>(p.C, b, 0) + group * p.n;
        float h[4] = {}, a[4] = {}, bb[4] = {}, cc[4] = {};
        if (p.vec4) {
            if (n0 < p.n) {
                const float4 v = *reinterpret_cast<const float4*>(st + n0), w = *reinterpret_cast<const float4*>(A + n0);
                h[0] = v.x, h[1] = v.y, h[2] = v.z, h[3] = v.w;
                a[0] = w.x, a[1] = w.y, a[2] = w.z, a[3] = w.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < p.n)
                    h[i] = st[n0 + i], a[i] = A[n0 + i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n0 + i < p.n)
                bb[i] = to_f(B[n0 + i]), cc[i] = to_f(C[n0 + i]);
        x = to_f(row_ptr<const T>(p.x, b, 0)[c]);
        float step = to_f(row_ptr<const T>(p.delta, b, 0)[c]) + (p.delta_bias ? p.delta_bias[c] : 0.f);
        if (p.softplus)
            step = softplus(step);
        const float v = step * x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = fmaf(ex2(step * (a[i] * kLog2e)), h[i], v * bb[i]);
            y[0] = fmaf(h[i], cc[i], y[0]);
        }
        if (p.vec4) {
            if (n0 < p.n)
                *reinterpret_cast<float4*>(st + n0) = make_float4(h[0], h[1], h[2], h[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < p.n)
                    st[n0 + i] = h[i];
        }
    }
    group_sums<1, LANES, 1>(y, tid);
    if (have && sub == 0) {
        float v = fmaf(p.D ? p.D[c] : 0.f, x, y[0]);
        if (p.z.ptr)
            v *= silu(to_f(row_ptr<const T>(p.z, b, 0)[c]));
        row_ptr<T>(p.y, b, 0)[c] = from_f<T>(v);
    }
}

} // namespace sscan
} // namespace ttc
