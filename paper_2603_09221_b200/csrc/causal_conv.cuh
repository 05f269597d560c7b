// Depthwise causal convolution of token rows, z_t = bias + sum_j w_j x_{t-(W-1)+j}, y_t = act(z_t), its gradients, and the
// step of a single token.
//
// A thread owns V = 2 neighbouring channels (four in the step), loaded and stored at once where rows are aligned for it and
// one by one where they are not, computes on packed pairs of them, and walks over a tile of tokens with the
// last W inputs in registers, so an input is read once apart from the W - 1 rows in front of a tile.  Memory bounds all
// three kernels: one read and one write per element forward, two and one backward.
//
// Forward, 4 x 2048 tokens of 4096 channels, bfloat16, four taps, SiLU: 34.8 us, 3.9 TB/s (a copy of the same arrays by torch: 24.7);
// at four times the tokens 110 us, 4.9 TB/s.  Issue slots (62 %) are close behind; four channels to a thread 36.0, the next tokens'
// loads under way beside the arithmetic 38 (registers).  Backward, 8191 packed rows of 2047 channels, which allow accesses of
// two bytes only: 46 us, 50 instructions per element in 61 % of the issue slots; aligned, 4 x 2048 of 4096: 62.8 us, 3.2 TB/s.
// A step, 64 sequences of 4096 channels: 2.3 us.
#pragma once

#include <type_traits>

#include "block_common.cuh"

namespace ttc {
namespace conv {

using namespace blk;

constexpr int kThreads = 128;
constexpr int kAhead = 8, kGradAhead = 4;      // tokens whose loads are under way together

struct ConvDev {
    Seqs seqs;
    int d, act;
    int tile;                       // tokens of a tile
    int vec_w;                      // taps can be read by 16 bytes
    long long tiles;                // tiles of a sequence (equal) or of all rows (packed)
    long long all_tiles;
    Rows x, y, dy, dx;
    const float *w, *bias;
    const void *state, *dstate_out;
    void *state_out, *dstate;
    float *part;                    // [tiles in all][W + 1][d]: partial sums of dw and dbias
    float *dw, *dbias;
};

// The part of a sequence that lies in a tile of rows.
struct Segment {
    long long seq, row0, len;       // sequence, row of its first token, its length
    long long t0, t1;               // tokens of it in the tile
};

// First sequence that ends behind the first row of tile `i`.  Every lane of the warp looks at a place of its own, so that a
// round of loads narrows the search to a 32nd (up to 32 sequences: one round).  All lanes of the warp take part.
__device__ __forceinline__ long long first_sequence(const ConvDev& p, long long i)
{
    if (!p.seqs.offsets)
        return 0;
    const long long r0 = i * p.tile;
    long long lo = 0, hi = p.seqs.batch;
    while (lo < hi) {
        const long long step = (hi - lo + 31) / 32, b = lo + threadIdx.x % 32 * step;
        const bool before = b < hi && clamp_offset(p.seqs, b + 1) <= r0;
        const int count = __popc(__ballot_sync(0xffffffffu, before));
        if (count == 0)
            break;
        hi = lo + count * step < hi ? lo + count * step : hi;
        lo += (count - 1) * step + 1;
    }
    return lo;
}

// Calls f for every sequence that has tokens in tile `i`, the first of which may be `from`.
template <typename F> __device__ __forceinline__ void for_segments(const ConvDev& p, long long i, long long from, F&& f)
{
    if (!p.seqs.offsets) {
        const long long seq = i / p.tiles, t0 = (i % p.tiles) * p.tile;
        f(Segment{seq, 0, p.seqs.tokens, t0, t0 + p.tile < p.seqs.tokens ? t0 + p.tile : p.seqs.tokens});
        return;
    }
    const long long r0 = i * p.tile, r1 = r0 + p.tile < p.seqs.tokens ? r0 + p.tile : p.seqs.tokens;
    for (long long b = from; b < p.seqs.batch; ++b) {
        const Span s = span_of(p.seqs, b);
        if (s.row0 >= r1)
            break;
        const long long t0 = r0 > s.row0 ? r0 - s.row0 : 0, t1 = r1 - s.row0 < s.len ? r1 - s.row0 : s.len;
        if (t0 < t1)
            f(Segment{b, s.row0, s.len, t0, t1});
    }
}

// V channels of a row, `count` of which exist; ALIGNED: as one access.  What does not exist reads as the channel before it.
template <bool ALIGNED, typename T, int V> __device__ __forceinline__ Vec<T, V> fetch(const T* from, int count)
{
    if constexpr (ALIGNED) {
        return *reinterpret_cast<const Vec<T, V>*>(from);
    } else {
        static_assert(V == 2, "");
        Vec<T, V> r;
        r.v[0] = from[0];
        r.v[1] = from[count - 1];
        return r;
    }
}
template <bool ALIGNED, typename T, int V> __device__ __forceinline__ Vec<T, V> fetch_if(const T* from, bool ok, int count)
{
    if constexpr (ALIGNED) {
        return load_if(reinterpret_cast<const Vec<T, V>*>(from), ok);
    } else {
        Vec<T, V> r;
        r.v[0] = load_if(reinterpret_cast<const Vec<T, 1>*>(from), ok).v[0];
        r.v[1] = load_if(reinterpret_cast<const Vec<T, 1>*>(from + (count - 1)), ok).v[0];
        return r;
    }
}
template <bool ALIGNED, typename T, int V> __device__ __forceinline__ void give(T* to, const Vec<T, V>& v, int count)
{
    if constexpr (ALIGNED) {
        *reinterpret_cast<Vec<T, V>*>(to) = v;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < count)
                to[i] = v.v[i];
    }
}
template <typename T, int V> __device__ __forceinline__ void widen(f2 (&to)[V / 2], const Vec<T, V>& v)
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i)
        to[i] = pack2(to_f(v.v[2 * i]), to_f(v.v[2 * i + 1]));
}
template <typename T, int V> __device__ __forceinline__ Vec<T, V> narrow(const f2 (&from)[V / 2])
{
    Vec<T, V> r;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        float a, b;
        unpack2(from[i], a, b);
        r.v[2 * i] = from_f<T>(a), r.v[2 * i + 1] = from_f<T>(b);
    }
    return r;
}

template <typename T, int V, int W> struct Taps {
    f2 w[W][V / 2], b[V / 2];
    int count;                      // channels that exist
    __device__ __forceinline__ void load(const ConvDev& p, int c)
    {
        count = p.d - c < V ? p.d - c : V;
        float all[V * W], bias[V];
        const float* from = p.w + (long long)c * W;
        if (V * W % 4 == 0 && p.vec_w && count == V) {
#pragma unroll
            for (int i = 0; i < V * W; i += 4) {
                const float4 u = *reinterpret_cast<const float4*>(from + i);
                all[i] = u.x, all[i + 1] = u.y, all[i + 2] = u.z, all[i + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V * W; ++i)
                all[i] = i < count * W ? from[i] : 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            bias[v] = p.bias && v < count ? p.bias[c + v] : 0.f;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            b[i] = pack2(bias[2 * i], bias[2 * i + 1]);
#pragma unroll
            for (int j = 0; j < W; ++j)
                w[j][i] = pack2(all[2 * i * W + j], all[(2 * i + 1) * W + j]);
        }
    }
    // moves the window on by one input and returns z of pair i
    __device__ __forceinline__ f2 next(f2 (&in)[W][V / 2], int i, f2 x) const
    {
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
            in[j][i] = in[j + 1][i];
        in[W - 1][i] = x;
        f2 z = b[i];
#pragma unroll
        for (int j = 0; j < W; ++j)
            z = fma2(w[j][i], in[j][i], z);
        return z;
    }
};

// Input at token t of a sequence, which lies in the window in front of it where t < 0.
template <bool ALIGNED, typename T, int V, int W>
__device__ __forceinline__ Vec<T, V> input_at(const ConvDev& p, const Segment& s, long long t, int c, int count)
{
    const T* from = t >= 0 ? row_ptr<const T>(p.x, s.seq, s.row0 + t) + c : static_cast<const T*>(p.state) + (s.seq * (W - 1) + (W - 1) + t) * p.d + c;
    return fetch_if<ALIGNED, T, V>(from, t >= 0 || p.state, count);
}

// The last W - 1 inputs of sequence `seq`, channel c.
template <typename T, int W> __device__ __forceinline__ void keep_window(const ConvDev& p, long long seq, int c)
{
    const Span s = span_of(p.seqs, seq);
    const Segment g{seq, s.row0, s.len, 0, 0};
    T v[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        v[j] = input_at<true, T, 1, W>(p, g, s.len - (W - 1) + j, c, 1).v[0];
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        static_cast<T*>(p.state_out)[(seq * (W - 1) + j) * p.d + c] = v[j];
}
// In a launch of its own where state_out is state, behind the one that reads the windows in front.
template <typename T, int W> __global__ void __launch_bounds__(kThreads) conv_window_kernel(const ConvDev p)
{
    wait_for_previous();
    const int c = blockIdx.y * kThreads + threadIdx.x;
    if (c < p.d)
        keep_window<T, W>(p, blockIdx.x, c);
}

// Blocks past the tiles keep the last windows, one sequence each.
template <typename T, int V, bool ALIGNED, int W>
__global__ void __launch_bounds__(kThreads, 10) conv_kernel(const ConvDev p)
{
    const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
    if (blockIdx.x >= p.all_tiles) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c + i < p.d)
                keep_window<T, W>(p, blockIdx.x - p.all_tiles, c + i);
        return;
    }
    const long long from = first_sequence(p, blockIdx.x);
    if (c >= p.d)
        return;
    Taps<T, V, W> k;
    k.load(p, c);
    for_segments(p, blockIdx.x, from, [&](const Segment& s) {
        f2 in[W][V / 2];                                             // the last W inputs, oldest first
#pragma unroll
        for (int j = 1; j < W; ++j)
            widen(in[j], input_at<ALIGNED, T, V, W>(p, s, s.t0 - W + j, c, k.count));
        const T* x = row_ptr<const T>(p.x, s.seq, s.row0 + s.t0) + c;
        T* y = row_ptr<T>(p.y, s.seq, s.row0 + s.t0) + c;
        auto token = [&](const Vec<T, V>& v) {
            f2 out[V / 2], now[V / 2];
            widen(now, v);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const f2 z = k.next(in, i, now[i]);
                out[i] = p.act == TTC_ACT_SILU ? silu2(z) : z;
            }
            give<ALIGNED>(y, narrow<T, V>(out), k.count);
            y += p.y.ts;
        };
        int left = static_cast<int>(s.t1 - s.t0);
        for (; left >= kAhead; left -= kAhead) {
            Vec<T, V> now[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a, x += p.x.ts)
                now[a] = fetch<ALIGNED, T, V>(x, k.count);
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
                token(now[a]);
        }
        for (; left > 0; --left, x += p.x.ts)
            token(fetch<ALIGNED, T, V>(x, k.count));
    });
}

template <typename T, int V, bool ALIGNED, int W>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(const ConvDev p)
{
    wait_for_previous();
    const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
    if (c >= p.d)
        return;
    const long long b = blockIdx.x;
    const int count = p.d - c < V ? p.d - c : V;
    Vec<T, V> in[W];
    T* st = static_cast<T*>(p.state_out) + b * (W - 1) * p.d + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        in[j] = fetch<ALIGNED, T, V>(st + (long long)j * p.d, count);
    in[W - 1] = fetch<ALIGNED, T, V>(row_ptr<const T>(p.x, b, 0) + c, count);
    Taps<T, V, W> k;
    k.load(p, c);
    f2 z[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i)
        z[i] = k.b[i];
#pragma unroll
    for (int j = 0; j < W; ++j) {
        f2 now[V / 2];
        widen(now, in[j]);
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            z[i] = fma2(k.w[j][i], now[i], z[i]);
    }
    if (p.act == TTC_ACT_SILU)
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            z[i] = silu2(z[i]);
    give<ALIGNED>(row_ptr<T>(p.y, b, 0) + c, narrow<T, V>(z), count);
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        give<ALIGNED>(st + (long long)j * p.d, in[j + 1], count);
}

// Gradients.  With dz_t = dy_t act'(z_t):  dx_s = sum_j w_j dz_{s+W-1-j}, so a walk that has reached token t can give out
// the gradient of input t - (W - 1); it runs W - 1 tokens past its tile (whose z it computes again) or past the
// sequence's end (dz = 0), and in front of the sequence the inputs are the window's.
template <typename T, int V, bool ALIGNED, int W>
__global__ void __launch_bounds__(kThreads, 7) conv_grad_kernel(const ConvDev p)
{
    const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
    const long long from = first_sequence(p, blockIdx.x);
    if (c >= p.d)
        return;
    Taps<T, V, W> k;
    k.load(p, c);
    f2 dw[W][V / 2] = {}, db[V / 2] = {};
    for_segments(p, blockIdx.x, from, [&](const Segment& s) {
        f2 in[W][V / 2], dz[W][V / 2] = {};                          // the last W inputs and dz, oldest first
#pragma unroll
        for (int j = 1; j < W; ++j)
            widen(in[j], input_at<ALIGNED, T, V, W>(p, s, s.t0 - W + j, c, k.count));
        const T* x = row_ptr<const T>(p.x, s.seq, s.row0 + s.t0) + c;
        const T* dy = row_ptr<const T>(p.dy, s.seq, s.row0 + s.t0) + c;
        T* dx = p.dx.ptr ? row_ptr<T>(p.dx, s.seq, s.row0 + s.t0) + c : nullptr;
        // Token t: EDGE where it may lie past the tile or the sequence, or the input it leads to in front of the tile.
        auto token = [&](auto edge, long long u, const Vec<T, V>& vx, const Vec<T, V>& vy) {
            constexpr bool EDGE = decltype(edge)::value;
            const bool real = !EDGE || u < s.len, mine = !EDGE || u < s.t1;
            f2 now[V / 2], g[V / 2], out[V / 2] = {};
            const long long at = u - (W - 1), back = at - (s.len - (W - 1));          // input, and its place in the last window
            if (EDGE && back >= 0 && p.dstate_out)
                widen(out, fetch<ALIGNED, T, V>(static_cast<const T*>(p.dstate_out) + (s.seq * (W - 1) + back) * p.d + c, k.count));
            widen(now, vx);
            widen(g, vy);                                            // zero past the sequence
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const f2 z = k.next(in, i, now[i]);
                if (p.act == TTC_ACT_SILU) {
                    const f2 q = sigmoid2(z), rest = fma2(q, pack2(-1.f, -1.f), pack2(1.f, 1.f));
                    g[i] = real ? mul2(g[i], fma2(mul2(q, z), rest, q)) : 0;
                }
#pragma unroll
                for (int j = 0; j + 1 < W; ++j)
                    dz[j][i] = dz[j + 1][i];
                dz[W - 1][i] = g[i];
                if (mine) {
                    db[i] = add2(db[i], g[i]);
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        dw[j][i] = fma2(g[i], in[j][i], dw[j][i]);
                }
#pragma unroll
                for (int j = 0; j < W; ++j)
                    out[i] = fma2(k.w[j][i], dz[W - 1 - j][i], out[i]);
            }
            if (!EDGE || at >= s.t0) {
                if (dx) {
                    give<ALIGNED>(dx, narrow<T, V>(out), k.count);
                    dx += p.dx.ts;
                }
            } else if (s.t0 == 0 && p.dstate) {                      // of the window, by the tile that begins the sequence
                give<ALIGNED>(static_cast<T*>(p.dstate) + (s.seq * (W - 1) + (W - 1) + at) * p.d + c, narrow<T, V>(out), k.count);
            }
        };
        const long long stop = s.t1 + W - 1, rows = stop < s.len ? stop : s.len;
        // a group of W - 1 tokens, then groups that lie inside, then what is left
        auto edge = [&](long long t, int count) {
            Vec<T, V> vx[kGradAhead], vy[kGradAhead];
#pragma unroll
            for (int a = 0; a < kGradAhead; ++a) {
                const bool ok = a < count && t + a < rows;
                vx[a] = fetch_if<ALIGNED, T, V>(x + a * p.x.ts, ok, k.count);
                vy[a] = fetch_if<ALIGNED, T, V>(dy + a * p.dy.ts, ok, k.count);
            }
#pragma unroll
            for (int a = 0; a < kGradAhead; ++a)
                if (a < count)
                    token(std::true_type(), t + a, vx[a], vy[a]);
            x += count * p.x.ts, dy += count * p.dy.ts;
        };
        long long t = s.t0;
        int count = W - 1;                                           // not above kGradAhead
        for (;;) {
            edge(t, count);
            t += count;
            for (; t + kGradAhead <= s.t1; t += kGradAhead) {
                Vec<T, V> vx[kGradAhead], vy[kGradAhead];
#pragma unroll
                for (int a = 0; a < kGradAhead; ++a, x += p.x.ts, dy += p.dy.ts) {
                    vx[a] = fetch<ALIGNED, T, V>(x, k.count);
                    vy[a] = fetch<ALIGNED, T, V>(dy, k.count);
                }
#pragma unroll
                for (int a = 0; a < kGradAhead; ++a)
                    token(std::false_type(), t + a, vx[a], vy[a]);
            }
            if (t >= stop)
                break;
            count = stop - t < kGradAhead ? static_cast<int>(stop - t) : kGradAhead;
        }
    });
    if (p.part) {
        float* to = p.part + (long long)blockIdx.x * (W + 1) * p.d + c;
#pragma unroll
        for (int j = 0; j <= W; ++j)
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                float a, b;
                unpack2(j < W ? dw[j][i] : db[i], a, b);
                to[(long long)j * p.d + 2 * i] = a;
                if (2 * i + 1 < k.count)
                    to[(long long)j * p.d + 2 * i + 1] = b;
            }
    }
}

// Sums the tiles' shares of dw and dbias: a block per tap and 32 channels, the tiles dealt out to its eight warps, whose
// sums are added in a fixed order.  Blocks past the taps pass the gradient of the last window of a sequence without tokens
// on to its first one.
template <typename T, int W> __global__ void __launch_bounds__(256) conv_param_kernel(const ConvDev p)
{
    wait_for_previous();
    __shared__ float sum[8][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int c = blockIdx.x * 32 + lane, j = blockIdx.y;
    if (j > W) {
        const long long seq = j - (W + 1) + (long long)warp * (gridDim.y - (W + 1));
        if (c < p.d && seq < p.seqs.batch && span_of(p.seqs, seq).len == 0)
            for (int k = 0; k < W - 1; ++k) {
                const long long at = (seq * (W - 1) + k) * p.d + c;
                static_cast<T*>(p.dstate)[at] = p.dstate_out ? static_cast<const T*>(p.dstate_out)[at] : from_f<T>(0.f);
            }
        return;
    }
    if (!p.dw && !p.dbias)
        return;
    float s = 0.f;
    if (c < p.d)
        for (long long i = warp; i < p.all_tiles; i += 8)
            s += p.part[(i * (W + 1) + j) * p.d + c];
    sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < p.d) {
        for (int k = 1; k < 8; ++k)
            s += sum[k][lane];
        if (j < W) {
            if (p.dw)
                p.dw[(long long)c * W + j] = s;
        } else if (p.dbias) {
            p.dbias[c] = s;
        }
    }
}

} // namespace conv
} // namespace ttc
