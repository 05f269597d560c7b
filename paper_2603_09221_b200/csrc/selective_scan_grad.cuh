// Gradients of the selective state space scan (selective_scan.cuh).  With g_t = dy_t silu(z_t) and the co-states
//     q_t = C_t g_t + exp(D_{t+1} A) q_{t+1}
// both recurrences, h forward and q backward, have the same decays, and the product of a span's decays is exp(A sum D_t).
// Every sequence is cut into pieces of 16 tokens, as many as the registers of a thread hold states and decays for:
//   1  local_kernel    of every piece, from nothing: the state behind it, the co-state a_{t0} q_{t0} in front of it (in the
//                      same walk: the running product of decays times C_t g_t) and the sum of its D_t
//   2  join_kernel     along every sequence: the state that enters each piece, the co-state that comes back to it; dstate
//   3  piece_kernel    of every piece, from those: states forward, co-states backward, every gradient
//   4  reduce kernels  the blocks' shares of dA, dD, ddelta_bias and of dB, dC, in a fixed order
// Steps 1 and 3 run over all tokens at once, whatever the number of sequences and channels.  Two exponentials per state
// and token in all.  The layout of a block is that of the forward kernel.
#pragma once

#include "selective_scan.cuh"

namespace ttc {
namespace sscan {

constexpr int kGradThreads = 128;
constexpr int kPiece = 16;        // tokens of a piece
constexpr int kRun = 4;           // pieces that a block works through, one behind the other

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

template <typename T, int LANES> struct Tile {
    static constexpr int CH = kGradThreads / LANES, NP = LANES * 4, TB = kPiece;
    static constexpr int EPT = (TB * CH + kGradThreads - 1) / kGradThreads;
    static constexpr int BPT = (TB * NP + kGradThreads - 1) / kGradThreads;
    static constexpr int WARPS = kGradThreads / 32;
    static constexpr size_t smem_local() { return sizeof(float) * (TB * CH * 6 + TB * NP * 2); }
    // tokens (D, D, Dx, Dx | g, g), B, C, y and q . B and A . (q a h), shares of dB and dC by warp
    static constexpr size_t smem_piece() { return sizeof(float) * (TB * CH * 6 + TB * NP * 2 + TB * CH * 3 + WARPS * TB * NP * 2); }
};

// Decays and rows of a tile of kPiece tokens from token t of the run into shared memory.
template <typename T, int LANES> struct Loader {
    using S = Tile<T, LANES>;
    static constexpr int CH = S::CH, NP = S::NP, TB = S::TB, EPT = S::EPT, BPT = S::BPT;
    float x[EPT], dy[EPT], z[EPT], step[EPT];      // of this thread's tokens

    __device__ __forceinline__ void load(const GradDev& p, const Piece& q, long long t, int group, int chan, bool have_l, float bias,
                                         float4* s_tok, float2* s_g, float* s_B, float* s_C)
    {
        const int tid = threadIdx.x, lc = tid % CH, lt = tid / CH;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const int u = e * (kGradThreads / CH) + lt;
            const bool ok = have_l && u < TB && t + u < q.t1;
            x[e] = dy[e] = z[e] = step[e] = 0.f;
            if (ok) {
                const long long row = q.row0 + t + u;
                x[e] = to_f(row_ptr<const T>(p.f.x, q.seq, row)[chan]);
                step[e] = to_f(row_ptr<const T>(p.f.delta, q.seq, row)[chan]) + bias;
                dy[e] = to_f(row_ptr<const T>(p.dy, q.seq, row)[chan]);
                if (p.f.z.ptr)
                    z[e] = to_f(row_ptr<const T>(p.f.z, q.seq, row)[chan]);
            }
        }
#pragma unroll
        for (int e = 0; e < BPT; ++e) {
            const int at = e * kGradThreads + tid, u = at / NP, k = at % NP;
            float b = 0.f, c = 0.f;
            if (u < TB && t + u < q.t1 && k < p.f.n) {
                b = to_f(row_ptr<const T>(p.f.B, q.seq, q.row0 + t + u)[group * p.f.n + k]);
                c = to_f(row_ptr<const T>(p.f.C, q.seq, q.row0 + t + u)[group * p.f.n + k]);
            }
            if (at < TB * NP)
                s_B[at] = b, s_C[at] = c;
        }
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const int u = e * (kGradThreads / CH) + lt;
            const bool ok = have_l && u < TB && t + u < q.t1;
            if (ok && p.f.softplus)
                step[e] = softplus(step[e]);
            const float v = ok ? step[e] * x[e] : 0.f;
            const float g = p.f.z.ptr && ok ? dy[e] * silu(z[e]) : dy[e];
            if (u < TB) {
                s_tok[u * CH + lc] = make_float4(step[e], step[e], v, v);
                s_g[u * CH + lc] = make_float2(g, g);
            }
        }
    }
};

template <typename T, int LANES>
__global__ void __launch_bounds__(kGradThreads) grad_local_kernel(const GradDev p)
{
    using S = Tile<T, LANES>;
    constexpr int CH = S::CH, NP = S::NP, TB = S::TB;
    extern __shared__ float4 smem[];
    float4* s_tok = smem;
    float* s_B = reinterpret_cast<float*>(s_tok + TB * CH);
    float* s_C = s_B + TB * NP;
    float2* s_g = reinterpret_cast<float2*>(s_C + TB * NP);

    Piece q;
    if (!find_piece(p.f, blockIdx.x, q))
        return;
    const int tid = threadIdx.x, sub = tid % LANES, ch = tid / LANES;
    const int group = blockIdx.y / p.f.chan_blocks, per_group = p.f.d / p.f.groups;
    const int c0 = (blockIdx.y % p.f.chan_blocks) * CH;
    const int my = group * per_group + c0 + ch, n0 = sub * 4;
    const bool have = c0 + ch < per_group;
    const int chan = group * per_group + c0 + tid % CH;
    const bool have_l = c0 + tid % CH < per_group;
    f2 A2[2];
    {
        float a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = have && n0 + i < p.f.n ? p.f.A[(long long)my * p.f.n + n0 + i] * kLog2e : 0.f;
        A2[0] = pack2(a[0], a[1]), A2[1] = pack2(a[2], a[3]);
    }
    const float bias = p.f.delta_bias && have_l ? p.f.delta_bias[chan] : 0.f;
    Loader<T, LANES> tile;
    for (int k = 0; k < kRun; ++k) {
        const long long t = q.t0 + k * kPiece;
        if (t >= q.t1)
            break;
        __syncthreads();
        tile.load(p, q, t, group, chan, have_l, bias, s_tok, s_g, s_B, s_C);
        __syncthreads();
        f2 h2[2] = {0, 0}, r2[2] = {0, 0}, prod[2];
        prod[0] = prod[1] = pack2(1.f, 1.f);
        float total = 0.f;
#pragma unroll 4
        for (int u = 0; u < TB; ++u) {
            const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[u * CH + ch];
            const f2 g = reinterpret_cast<const f2*>(s_g)[u * CH + ch];
            const ulonglong2 b = reinterpret_cast<const ulonglong2*>(s_B)[u * LANES + sub];
            const ulonglong2 c = reinterpret_cast<const ulonglong2*>(s_C)[u * LANES + sub];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float e0, e1;
                unpack2(mul2(A2[i], tok.x), e0, e1);
                const f2 a = pack2(ex2(e0), ex2(e1));
                h2[i] = fma2(a, h2[i], mul2(tok.y, i ? b.y : b.x));
                prod[i] = mul2(prod[i], a);
                r2[i] = fma2(prod[i], mul2(g, i ? c.y : c.x), r2[i]);
            }
            float s, s1;
            unpack2(tok.x, s, s1);
            total += s;
        }
        const long long slot = (long long)blockIdx.x * kRun + k;
        float h[4], r[4];
        unpack2(h2[0], h[0], h[1]);
        unpack2(h2[1], h[2], h[3]);
        unpack2(r2[0], r[0], r[1]);
        unpack2(r2[1], r[2], r[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (have && n0 + i < p.f.n) {
                p.h[(slot * p.f.d + my) * p.f.n + n0 + i] = h[i];
                p.r[(slot * p.f.d + my) * p.f.n + n0 + i] = r[i];
            }
        if (have && sub == 0)
            p.step[slot * p.f.d + my] = total;
    }
}

// blockIdx.z 0: states forward, 1: co-states backward.  In: what each piece adds; out: what enters it.
static __global__ void __launch_bounds__(128) grad_join_kernel(const GradDev p)
{
    const long long at = (long long)blockIdx.y * 128 + threadIdx.x, size = (long long)p.f.d * p.f.n;
    if (at >= size)
        return;
    const long long seq = blockIdx.x, c = at / p.f.n;
    const long long first = (p.f.piece_map ? p.f.seq_first[seq] : seq * p.f.pieces_per_seq) * kRun;
    const long long most = p.f.piece_map ? (p.f.seq_first[seq + 1] * (long long)kRun - first) : p.f.pieces_per_seq * kRun;
    long long count = (span_of(p.f.seqs, seq).len + kPiece - 1) / kPiece;
    count = count < most ? count : most;
    const float a = p.f.A[at] * kLog2e;
    constexpr int kAhead = 8;
    if (blockIdx.z == 0) {
        float h = p.f.state ? p.f.state[seq * size + at] : 0.f;
        for (long long k = 0; k < count; k += kAhead) {
            float v[kAhead], s[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (k + i < count)
                    v[i] = p.h[(first + k + i) * size + at], s[i] = p.step[(first + k + i) * p.f.d + c];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (k + i < count) {
                    p.h[(first + k + i) * size + at] = h;
                    h = fmaf(ex2(a * s[i]), h, v[i]);
                }
        }
    } else {
        float r = p.dstate_out ? p.dstate_out[seq * size + at] : 0.f;
        for (long long k = count - 1; k >= 0; k -= kAhead) {
            float v[kAhead], s[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (k - i >= 0)
                    v[i] = p.r[(first + k - i) * size + at], s[i] = p.step[(first + k - i) * p.f.d + c];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (k - i >= 0) {
                    p.r[(first + k - i) * size + at] = r;
                    r = fmaf(ex2(a * s[i]), r, v[i]);
                }
        }
        if (p.dstate)
            p.dstate[seq * size + at] = r;
    }
}

template <typename T, int LANES>
__global__ void __launch_bounds__(kGradThreads, 2) grad_piece_kernel(const GradDev p)
{
    using S = Tile<T, LANES>;
    constexpr int CH = S::CH, NP = S::NP, TB = S::TB, EPT = S::EPT, WARPS = S::WARPS;
    extern __shared__ float4 smem[];
    float4* s_tok = smem;
    float* s_B = reinterpret_cast<float*>(s_tok + TB * CH);
    float* s_C = s_B + TB * NP;
    float2* s_g = reinterpret_cast<float2*>(s_C + TB * NP);
    float* s_y = reinterpret_cast<float*>(s_g + TB * CH);            // C . h
    float2* s_q = reinterpret_cast<float2*>(s_y + TB * CH);          // q . B and A . (q a h)
    float* s_BC = reinterpret_cast<float*>(s_q + TB * CH);           // [WARPS][TB][2][NP]

    Piece q;
    if (!find_piece(p.f, blockIdx.x, q))
        return;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, sub = tid % LANES, ch = tid / LANES;
    const int group = blockIdx.y / p.f.chan_blocks, per_group = p.f.d / p.f.groups, block = blockIdx.y % p.f.chan_blocks;
    const int c0 = block * CH;
    const int my = group * per_group + c0 + ch, n0 = sub * 4;
    const bool have = c0 + ch < per_group;
    const int lc = tid % CH, lt = tid / CH, chan = group * per_group + c0 + lc;
    const bool have_l = c0 + lc < per_group;
    f2 A2[2], dA2[2] = {0, 0};
    {
        float a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = have && n0 + i < p.f.n ? p.f.A[(long long)my * p.f.n + n0 + i] * kLog2e : 0.f;
        A2[0] = pack2(a[0], a[1]), A2[1] = pack2(a[2], a[3]);
    }
    const float bias = p.f.delta_bias && have_l ? p.f.delta_bias[chan] : 0.f;
    const float skip = p.f.D && have_l ? p.f.D[chan] : 0.f;
    float sum_D = 0.f, sum_bias = 0.f;
    Loader<T, LANES> tile;
    for (int k = 0; k < kRun; ++k) {
        const long long t = q.t0 + k * kPiece;
        if (t >= q.t1)
            break;
        const long long slot = (long long)blockIdx.x * kRun + k;
        float h[4], r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = r[i] = 0.f;
            if (have && n0 + i < p.f.n) {
                h[i] = p.h[(slot * p.f.d + my) * p.f.n + n0 + i];
                r[i] = p.r[(slot * p.f.d + my) * p.f.n + n0 + i];
            }
        }
        __syncthreads();
        tile.load(p, q, t, group, chan, have_l, bias, s_tok, s_g, s_B, s_C);
        __syncthreads();
        f2 a2[TB][2], h2[TB + 1][2], r2[2];                          // h2[u]: the state in front of token u
        h2[0][0] = pack2(h[0], h[1]), h2[0][1] = pack2(h[2], h[3]);
        r2[0] = pack2(r[0], r[1]), r2[1] = pack2(r[2], r[3]);
#pragma unroll
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
                    a2[u + j][i] = pack2(ex2(e0), ex2(e1));
                    h2[u + j + 1][i] = fma2(a2[u + j][i], h2[u + j][i], mul2(tok.y, i ? b.y : b.x));
                }
                if (p.dz.ptr) {
                    const ulonglong2 c = reinterpret_cast<const ulonglong2*>(s_C)[(u + j) * LANES + sub];
                    y2 = fma2(h2[u + j + 1][1], c.y, mul2(h2[u + j + 1][0], c.x));
                }
                part[j] = sum2(y2);
            }
            if (p.dz.ptr) {
                group_sums<4, LANES, 1>(part, lane);
                constexpr int left = LANES >= 4 ? 1 : 4 / LANES;
                const int first = first_value<4, LANES>(sub);
                if (LANES <= 4 || sub < 4)
#pragma unroll
                    for (int i = 0; i < left; ++i)
                        s_y[(u + first + i) * CH + ch] = part[i];
            }
        }
        float pair[4];                                               // q . B and A . (q a h) of two tokens
#pragma unroll
        for (int u = TB - 1; u >= 0; --u) {
            const ulonglong2 tok = reinterpret_cast<const ulonglong2*>(s_tok)[u * CH + ch];
            const f2 g = reinterpret_cast<const f2*>(s_g)[u * CH + ch];
            const ulonglong2 b = reinterpret_cast<const ulonglong2*>(s_B)[u * LANES + sub];
            const ulonglong2 c = reinterpret_cast<const ulonglong2*>(s_C)[u * LANES + sub];
            float bc[8];
            f2 qB = 0, through = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f2 co = fma2(g, i ? c.y : c.x, r2[i]);         // q_t
                unpack2(mul2(co, tok.y), bc[2 * i], bc[2 * i + 1]);
                unpack2(mul2(h2[u + 1][i], g), bc[4 + 2 * i], bc[5 + 2 * i]);
                r2[i] = mul2(a2[u][i], co);
                const f2 qah = mul2(r2[i], h2[u][i]);
                dA2[i] = fma2(tok.x, qah, dA2[i]);
                qB = i ? fma2(co, b.y, qB) : mul2(co, b.x);
                through = i ? fma2(A2[i], qah, through) : mul2(A2[i], qah);
            }
            group_sums<8, 32 / LANES, LANES>(bc, lane);
            {
                constexpr int W = 32 / LANES, left = W >= 8 ? 1 : 8 / W;
                const int j = lane / LANES, first = first_value<8, W>(j);
                if (W <= 8 || j < 8)
#pragma unroll
                    for (int i = 0; i < left; ++i) {
                        const int v = first + i;
                        s_BC[((warp * TB + u) * 2 + v / 4) * NP + n0 + v % 4] = bc[i];
                    }
            }
            pair[(u & 1) * 2] = sum2(qB);
            pair[(u & 1) * 2 + 1] = sum2(through);
            if (u % 2 == 0) {
                group_sums<4, LANES, 1>(pair, lane);
                constexpr int left = LANES >= 4 ? 1 : 4 / LANES;
                const int first = first_value<4, LANES>(sub);
                if (LANES <= 4 || sub < 4)
#pragma unroll
                    for (int i = 0; i < left; ++i)
                        reinterpret_cast<float*>(s_q)[((u + (first + i) / 2) * CH + ch) * 2 + (first + i) % 2] = pair[i];
            }
        }
        __syncthreads();
        // shares of dB and dC of this block's channels
        if (p.part_BC) {
            const long long row = slot * kPiece, rows = p.runs * kRun * kPiece;
            float* to = p.part_BC + (((long long)block * rows + row) * p.f.groups + group) * 2 * NP;
            for (int at = tid; at < TB * 2 * NP; at += kGradThreads) {
                const int u = at / (2 * NP), v = at % (2 * NP);
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < WARPS; ++w)
                    s += s_BC[(w * TB + u) * 2 * NP + v];
                to[(long long)u * p.f.groups * 2 * NP + v] = s;
            }
        }
        // gradients of this thread's tokens
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const int u = e * (kGradThreads / CH) + lt;
            if (u >= TB || t + u >= q.t1 || !have_l)
                continue;
            const long long row = q.row0 + t + u;
            const float2 s = s_q[u * CH + lc];
            const float g = s_g[u * CH + lc].x;
            if (p.dx.ptr)
                row_ptr<T>(p.dx, q.seq, row)[chan] = from_f<T>(fmaf(tile.step[e], s.x, skip * g));
            float dstep = fmaf(tile.x[e], s.x, s.y * (1.f / kLog2e));
            if (p.f.softplus)
                dstep *= -expm1f(-tile.step[e]);                     // the logistic function of what the softplus was given
            if (p.ddelta.ptr)
                row_ptr<T>(p.ddelta, q.seq, row)[chan] = from_f<T>(dstep);
            if (p.dz.ptr)
                row_ptr<T>(p.dz, q.seq, row)[chan] = from_f<T>(tile.dy[e] * fmaf(skip, tile.x[e], s_y[u * CH + lc]) * silu_slope(tile.z[e]));
            sum_D = fmaf(g, tile.x[e], sum_D);
            sum_bias += dstep;
        }
    }
    if (p.part_A) {
        float v[4];
        unpack2(dA2[0], v[0], v[1]);
        unpack2(dA2[1], v[2], v[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (have && n0 + i < p.f.n)
                p.part_A[((long long)blockIdx.x * p.f.d + my) * p.f.n + n0 + i] = v[i];
    }
    if (p.part_D) {
        __syncthreads();
        float2* sums = reinterpret_cast<float2*>(s_tok);
        sums[tid] = make_float2(sum_D, sum_bias);
        __syncthreads();
        if (tid < CH && have_l) {
            float a = 0.f, b = 0.f;
            for (int i = tid; i < kGradThreads; i += CH)
                a += sums[i].x, b += sums[i].y;
            p.part_D[((long long)blockIdx.x * 2) * p.f.d + chan] = a;
            p.part_D[((long long)blockIdx.x * 2 + 1) * p.f.d + chan] = b;
        }
    }
}

// Sum over the runs: out[i] = sum_r part[r * stride + i], i < size; runs without a sequence were not written.
static __global__ void __launch_bounds__(256) grad_sum_kernel(const GradDev p, const float* part, long long stride, long long size, float* out)
{
    __shared__ float sum[8][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const long long i = (long long)blockIdx.x * 32 + lane;
    const long long runs = p.f.piece_map ? p.f.seq_first[p.f.seqs.batch] : p.runs;
    float s = 0.f;
    if (i < size)
        for (long long r = warp; r < runs; r += 8)
            s += part[r * stride + i];
    sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && i < size) {
        for (int k = 1; k < 8; ++k)
            s += sum[k][lane];
        out[i] = s;
    }
}

// dB and dC of every token: the channel blocks of its group added up.
template <typename T> __global__ void __launch_bounds__(256) grad_rows_kernel(const GradDev p, int NP)
{
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
