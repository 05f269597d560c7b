// Depthwise causal convolution of token rows, z_t = bias + sum_j w_j x_{t-(W-1)+j}, y_t = act(z_t), its gradients, and the
// step of a single token.
//
// A thread owns V neighbouring channels (8 bytes, backward 4, where rows are aligned for it) and walks over a tile of tokens with the
// last W inputs in registers, so an input is read once apart from the W - 1 rows in front of a tile.  Memory bounds all
// three kernels: one read and one write per element forward, two and one backward.
#pragma once

#include "block_common.cuh"

namespace ttc {
namespace conv {

using namespace blk;

constexpr int kThreads = 128;

struct ConvDev {
    Seqs seqs;
    int d, act;
    int tile;                       // tokens of a tile
    int vec_w;                      // taps can be read by 16 bytes
    long long tiles;                // tiles of a sequence (equal) or of all rows (packed)
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

// Calls f for every sequence that has tokens in tile `i`.
template <typename F> __device__ __forceinline__ void for_segments(const ConvDev& p, long long i, F&& f)
{
    if (!p.seqs.offsets) {
        const long long seq = i / p.tiles, t0 = (i % p.tiles) * p.tile;
        f(Segment{seq, 0, p.seqs.tokens, t0, t0 + p.tile < p.seqs.tokens ? t0 + p.tile : p.seqs.tokens});
        return;
    }
    const long long r0 = i * p.tile, r1 = r0 + p.tile < p.seqs.tokens ? r0 + p.tile : p.seqs.tokens;
    long long lo = 0, hi = p.seqs.batch;            // first sequence that ends behind r0
    while (lo < hi) {
        const long long mid = (lo + hi) / 2;
        if (clamp_offset(p.seqs, mid + 1) > r0)
            hi = mid;
        else
            lo = mid + 1;
    }
    for (; lo < p.seqs.batch; ++lo) {
        const Span s = span_of(p.seqs, lo);
        if (s.row0 >= r1)
            break;
        const long long t0 = r0 > s.row0 ? r0 - s.row0 : 0, t1 = r1 - s.row0 < s.len ? r1 - s.row0 : s.len;
        if (t0 < t1)
            f(Segment{lo, s.row0, s.len, t0, t1});
    }
}

template <typename T, int V, int W> struct Taps {
    float w[W][V], b[V];
    __device__ __forceinline__ void load(const ConvDev& p, int c)
    {
        float all[V * W];
        const float* from = p.w + (long long)c * W;
        if (V * W % 4 == 0 && p.vec_w) {
#pragma unroll
            for (int i = 0; i < V * W; i += 4) {
                const float4 u = *reinterpret_cast<const float4*>(from + i);
                all[i] = u.x, all[i + 1] = u.y, all[i + 2] = u.z, all[i + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V * W; ++i)
                all[i] = from[i];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            b[v] = p.bias ? p.bias[c + v] : 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j)
                w[j][v] = all[v * W + j];
        }
    }
    // moves the window on by one input and returns z of channel i
    __device__ __forceinline__ float next(float (&in)[W][V], int i, float x) const
    {
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
            in[j][i] = in[j + 1][i];
        in[W - 1][i] = x;
        float z = b[i];
#pragma unroll
        for (int j = 0; j < W; ++j)
            z = fmaf(w[j][i], in[j][i], z);
        return z;
    }
};

// Input at token t of a sequence, which lies in the window in front of it where t < 0.
template <typename T, int V, int W>
__device__ __forceinline__ Vec<T, V> input_at(const ConvDev& p, const Segment& s, long long t, int c)
{
    if (t >= 0)
        return *reinterpret_cast<const Vec<T, V>*>(row_ptr<const T>(p.x, s.seq, s.row0 + t) + c);
    if (p.state)
        return *reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.state) + (s.seq * (W - 1) + (W - 1) + t) * p.d + c);
    Vec<T, V> zero;
#pragma unroll
    for (int v = 0; v < V; ++v)
        zero.v[v] = from_f<T>(0.f);
    return zero;
}

constexpr int kAhead = 8;           // tokens whose loads are under way together

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads) conv_kernel(const ConvDev p)
{
    const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
    if (c >= p.d)
        return;
    Taps<T, V, W> k;
    k.load(p, c);
    for_segments(p, blockIdx.x, [&](const Segment& s) {
        float in[W][V];                                              // the last W inputs, oldest first
#pragma unroll
        for (int j = 1; j < W; ++j) {
            const Vec<T, V> v = input_at<T, V, W>(p, s, s.t0 - W + j, c);
#pragma unroll
            for (int i = 0; i < V; ++i)
                in[j][i] = to_f(v.v[i]);
        }
        const T* x = row_ptr<const T>(p.x, s.seq, s.row0 + s.t0) + c;
        T* y = row_ptr<T>(p.y, s.seq, s.row0 + s.t0) + c;
        auto give = [&](const Vec<T, V>& v, T* to) {
            Vec<T, V> out;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float z = k.next(in, i, to_f(v.v[i]));
                out.v[i] = from_f<T>(p.act == TTC_ACT_SILU ? silu(z) : z);
            }
            *reinterpret_cast<Vec<T, V>*>(to) = out;
        };
        int left = static_cast<int>(s.t1 - s.t0);
        for (; left >= kAhead; left -= kAhead, x += kAhead * p.x.ts, y += kAhead * p.y.ts) {
            Vec<T, V> next[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
                next[a] = *reinterpret_cast<const Vec<T, V>*>(x + a * p.x.ts);
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
                give(next[a], y + a * p.y.ts);
        }
        for (; left > 0; --left, x += p.x.ts, y += p.y.ts)
            give(*reinterpret_cast<const Vec<T, V>*>(x), y);
    });
}

// The last W - 1 inputs of every sequence.  A launch of its own, behind the one that reads the windows in front: state_out may be state.
template <typename T, int W>
__global__ void __launch_bounds__(kThreads) conv_window_kernel(const ConvDev p)
{
    const int c = blockIdx.y * kThreads + threadIdx.x;
    if (c >= p.d)
        return;
    const Span s = span_of(p.seqs, blockIdx.x);
    const Segment g{(long long)blockIdx.x, s.row0, s.len, 0, 0};
    T v[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        v[j] = input_at<T, 1, W>(p, g, s.len - (W - 1) + j, c).v[0];
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        static_cast<T*>(p.state_out)[((long long)blockIdx.x * (W - 1) + j) * p.d + c] = v[j];
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(const ConvDev p)
{
    const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
    if (c >= p.d)
        return;
    const long long b = blockIdx.x;
    Vec<T, V> in[W], out;
    T* st = static_cast<T*>(p.state_out) + b * (W - 1) * p.d + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        in[j] = *reinterpret_cast<const Vec<T, V>*>(st + (long long)j * p.d);
    in[W - 1] = *reinterpret_cast<const Vec<T, V>*>(row_ptr<const T>(p.x, b, 0) + c);
    Taps<T, V, W> k;
    k.load(p, c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float z = k.b[i];
#pragma unroll
        for (int j = 0; j < W; ++j)
            z = fmaf(k.w[j][i], to_f(in[j].v[i]), z);
        out.v[i] = from_f<T>(p.act == TTC_ACT_SILU ? silu(z) : z);
    }
    *reinterpret_cast<Vec<T, V>*>(row_ptr<T>(p.y, b, 0) + c) = out;
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        *reinterpret_cast<Vec<T, V>*>(st + (long long)j * p.d) = in[j + 1];
}

constexpr int kGradAhead = 8;

// Gradients.  With dz_t = dy_t act'(z_t):  dx_s = sum_j w_j dz_{s+W-1-j}, so a walk that has reached token t can give out
// the gradient of input t - (W - 1); it runs W - 1 tokens past its tile (whose z it computes again) or past the
// sequence's end (dz = 0), and in front of the sequence the inputs are the window's.
template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads) conv_grad_kernel(const ConvDev p)
{
    const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
    if (c >= p.d)
        return;
    Taps<T, V, W> k;
    k.load(p, c);
    float dw[W][V] = {}, db[V] = {};
    auto push = [](float (&dz)[W][V], int i, float g) {
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
            dz[j][i] = dz[j + 1][i];
        dz[W - 1][i] = g;
    };
    auto input_grad = [&](const float (&dz)[W][V], int i, float g) {
#pragma unroll
        for (int j = 0; j < W; ++j)
            g = fmaf(k.w[j][i], dz[W - 1 - j][i], g);
        return g;
    };
    for_segments(p, blockIdx.x, [&](const Segment& s) {
        float in[W][V], dz[W][V] = {};                               // the last W inputs and dz, oldest first
#pragma unroll
        for (int j = 1; j < W; ++j) {
            const Vec<T, V> v = input_at<T, V, W>(p, s, s.t0 - W + j, c);
#pragma unroll
            for (int i = 0; i < V; ++i)
                in[j][i] = to_f(v.v[i]);
        }
        // one token, wherever it lies
        auto any = [&](long long u) {
            const bool real = u < s.len, mine = u < s.t1;
            Vec<T, V> nx, ny, extra, out;
            if (real) {
                nx = *reinterpret_cast<const Vec<T, V>*>(row_ptr<const T>(p.x, s.seq, s.row0 + u) + c);
                ny = *reinterpret_cast<const Vec<T, V>*>(row_ptr<const T>(p.dy, s.seq, s.row0 + u) + c);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float z = k.next(in, i, real ? to_f(nx.v[i]) : 0.f);
                float g = real ? to_f(ny.v[i]) : 0.f;
                if (p.act == TTC_ACT_SILU && real)
                    g *= silu_slope(z);
                push(dz, i, g);
                if (mine) {
                    db[i] += g;
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        dw[j][i] = fmaf(g, in[j][i], dw[j][i]);
                }
            }
            // inputs of this tile, and of the window for the tile that begins the sequence
            const long long at = u - (W - 1);
            if (at < s.t0 && !(s.t0 == 0 && p.dstate))
                return;
            const long long back = at - (s.len - (W - 1));           // place in the last window
            const bool more = back >= 0 && p.dstate_out;
            if (more)
                extra = *reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(p.dstate_out) + (s.seq * (W - 1) + back) * p.d + c);
#pragma unroll
            for (int i = 0; i < V; ++i)
                out.v[i] = from_f<T>(input_grad(dz, i, more ? to_f(extra.v[i]) : 0.f));
            if (at < 0)
                *reinterpret_cast<Vec<T, V>*>(static_cast<T*>(p.dstate) + (s.seq * (W - 1) + (W - 1) + at) * p.d + c) = out;
            else if (p.dx.ptr)
                *reinterpret_cast<Vec<T, V>*>(row_ptr<T>(p.dx, s.seq, s.row0 + at) + c) = out;
        };
        const long long stop = s.t1 + W - 1;
        long long t = s.t0;
        for (; t < s.t0 + W - 1; ++t)
            any(t);
        // in between, a token and the input W - 1 in front of it are both of this tile, and the last window is further on
        const T* x = row_ptr<const T>(p.x, s.seq, s.row0 + t) + c;
        const T* dy = row_ptr<const T>(p.dy, s.seq, s.row0 + t) + c;
        T* dx = p.dx.ptr ? row_ptr<T>(p.dx, s.seq, s.row0 + t - (W - 1)) + c : nullptr;
        for (; t + kGradAhead <= s.t1; t += kGradAhead, x += kGradAhead * p.x.ts, dy += kGradAhead * p.dy.ts) {
            Vec<T, V> nx[kGradAhead], ny[kGradAhead];
#pragma unroll
            for (int a = 0; a < kGradAhead; ++a) {
                nx[a] = *reinterpret_cast<const Vec<T, V>*>(x + a * p.x.ts);
                ny[a] = *reinterpret_cast<const Vec<T, V>*>(dy + a * p.dy.ts);
            }
#pragma unroll
            for (int a = 0; a < kGradAhead; ++a) {
                Vec<T, V> out;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float z = k.next(in, i, to_f(nx[a].v[i]));
                    float g = to_f(ny[a].v[i]);
                    if (p.act == TTC_ACT_SILU)
                        g *= silu_slope(z);
                    push(dz, i, g);
                    db[i] += g;
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        dw[j][i] = fmaf(g, in[j][i], dw[j][i]);
                    out.v[i] = from_f<T>(input_grad(dz, i, 0.f));
                }
                if (dx) {
                    *reinterpret_cast<Vec<T, V>*>(dx) = out;
                    dx += p.dx.ts;
                }
            }
        }
        for (; t < stop; ++t)
            any(t);
    });
    if (p.part) {
        float* to = p.part + (long long)blockIdx.x * (W + 1) * p.d + c;
#pragma unroll
        for (int j = 0; j <= W; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i)
                to[(long long)j * p.d + i] = j < W ? dw[j][i] : db[i];
    }
}

// Sums the tiles' shares of dw and dbias: a block per tap and 32 channels, the tiles dealt out to its eight warps, whose
// sums are added in a fixed order.
template <int W> __global__ void __launch_bounds__(256) conv_param_kernel(const ConvDev p, long long tiles)
{
    __shared__ float sum[8][33];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int c = blockIdx.x * 32 + lane, j = blockIdx.y;
    float s = 0.f;
    if (c < p.d)
        for (long long i = warp; i < tiles; i += 8)
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

// Sequences without tokens: what the last window gets goes to the first one.
template <typename T, int W> __global__ void __launch_bounds__(kThreads) conv_empty_kernel(const ConvDev p)
{
    const int c = blockIdx.y * kThreads + threadIdx.x;
    if (c >= p.d || span_of(p.seqs, blockIdx.x).len > 0)
        return;
    for (int j = 0; j < W - 1; ++j) {
        const long long at = ((long long)blockIdx.x * (W - 1) + j) * p.d + c;
        static_cast<T*>(p.dstate)[at] = p.dstate_out ? static_cast<const T*>(p.dstate_out)[at] : from_f<T>(0.f);
    }
}

} // namespace conv
} // namespace ttc
