// Gradients of linear attention with a decay for each head.  With Z = dL/dS_C of a chunk (that of the state behind it) and q' = scale q:
//
//     dq_i = scale [ sum_{j <= i} exp(G_i - G_j) (dy_i . v_j) k_j + exp(G_i) S_0 dy_i ]
//     dk_j = sum_{i >= j} exp(G_i - G_j) (dy_i . v_j) q'_i + exp(R_j) Z v_j
//     dv_j = sum_{i >= j} exp(G_i - G_j) (q'_i . k_j) dy_i + exp(R_j) Z' k_j
//     dL/dS_0 = exp(G_C) Z + sum_i exp(G_i) q'_i dy_i'
//     dl_t = exp(G_C) <Z, S_0> + sum_{i >= t} e_i + sum_{j < t} f_j + sum_{i >= t > j} M_ij        (what passes through token t's decay)
//       e_i = exp(G_i) q'_i S_0 dy_i,   f_j = exp(R_j) k_j Z v_j,   M_ij = exp(G_i - G_j) (q'_i . k_j)(dy_i . v_j)
//
// The last sum is taken without sums that cancel: sum_{i >= t} (row_i - col_i) of M's row and column sums would do, but its rounding errors are those of all pairs
// behind t, of which only the few that span t count where decays are strong (dA was off by 4e-6 of its norm).  Instead, with the chunk in four blocks of 32: pairs within t's block
// one by one (prefix sums of M's rows, added up over the rows from t on); pairs of t's block and an earlier one by row sums, with a later one by column
// sums, and pairs of blocks on both sides of t's by their totals.
// dl goes into float32 sums over all tokens (dA, ddelta_bias): M is taken from the float32 scores, and S_0 and Z go into e and f as two numbers of 16 bits
// (2^-18 of the value).
//
// The states in front of the chunks come from a state walk, the Z from one that goes backwards along queries and dy; then one
// kernel finds dq, e and row, one dk, dv, f and col, and a small one dl.
#pragma once

#include "decay_attention.cuh"

namespace ttc {
namespace dattn {

__device__ __forceinline__ void load_image(uint32_t to, const char* from, int bytes)
{
    for (int i = threadIdx.x * 16; i < bytes; i += kThreads * 16)
        copy16(to + i, from + i, true);
}

struct GradDev {
    AttnDev f;
    Rows dy, dq, dk, dv, ddelta;
    int vec_dy, vec_dq, vec_dk, vec_dv;
    const float* dstate_out;
    float *dA, *dbias, *dstate;
    // scratch
    float *part_q, *part_k;                      // dq, dk of every head, where heads share them: [rows][heads][dk]
    char *image_S, *image_Z;                     // [chunks][heads][2][DV / 8][DK][8]
    float *unit_S, *unit_Z;
    float* tokens;                               // [5][heads][chunks][128]: e, row sums, f, column sums (both without the blocks on the diagonal), pairs within t's block
    float* bridges;                              // [chunks][heads][2]: of pairs on both sides of the second and the third block
    float* across;                               // exp(G_C) <Z, S_0>: [chunks][heads]
    float* sums;                                 // of dA and of ddelta_bias: [2][heads][chunks]
    int want_q, want_kv, want_l;
};

template <int DK, int DV> struct GradShape {
    static constexpr int K_BYTES = DK / 64 * kBox, V_BYTES = DV / 64 * kBox, IMAGE = DK * DV * 2;
    static constexpr int SMEM = 1024 + 2 * K_BYTES + 2 * V_BYTES + 2 * IMAGE;
};

// Half of a row of results (COLS / 2 of tensor memory's columns), times f, staged in a tile.
template <typename T, int COLS> __device__ __forceinline__ void stage_row(uint32_t from, char* tile, int row, int half, float f)
{
#pragma unroll
    for (int c0 = 0; c0 < COLS / 2; c0 += 32) {
        float v[32];
        tmem_ld32(from + half * (COLS / 2) + c0, v);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
            const uint4 w = make_uint4(pack16<T>(v[j] * f, v[j + 1] * f), pack16<T>(v[j + 2] * f, v[j + 3] * f), pack16<T>(v[j + 4] * f, v[j + 5] * f),
                                       pack16<T>(v[j + 6] * f, v[j + 7] * f));
            *reinterpret_cast<uint4*>(tile + tile_at(row, (half * (COLS / 2) + c0 + j) / 8)) = w;
        }
    }
}
// The same in float32, to the head's part of a sum over the heads of a group.
template <int COLS> __device__ __forceinline__ void part_row(uint32_t from, float* to, int width, bool ok, int half, float f)
{
#pragma unroll
    for (int c0 = 0; c0 < COLS / 2; c0 += 32) {
        float v[32];
        const int at = half * (COLS / 2) + c0;
        tmem_ld32(from + at, v);
        if (ok) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (at + j < width)
                    to[at + j] = v[j] * f;
        }
    }
}
// Half of a row of results, times f, back to where it was; returns its product with the same half of row `row` of a tile.
template <typename T, int COLS> __device__ __forceinline__ float weigh_row(uint32_t at, const char* tile, int row, int half, float f)
{
    float dot = 0.f;
#pragma unroll
    for (int c0 = 0; c0 < COLS / 2; c0 += 32) {
        float v[32];
        const uint32_t here = at + half * (COLS / 2) + c0;
        tmem_ld32(here, v);
#pragma unroll
        for (int j = 0; j < 32; ++j)
            v[j] *= f;
        if (tile) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                const uint4 w = *reinterpret_cast<const uint4*>(tile + tile_at(row, (half * (COLS / 2) + c0 + j) / 8));
                const uint32_t* u = &w.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 x = unpack16<T>(u[i]);
                    dot = fmaf(x.x, v[j + 2 * i], dot);
                    dot = fmaf(x.y, v[j + 2 * i + 1], dot);
                }
            }
        }
        tmem_st32(here, v);
    }
    return dot;
}

__device__ __forceinline__ long long packed_row(const AttnDev& p, const Chunk& c, int t) { return c.seq * p.seqs.tokens + c.row0 + t; }

// dq of one chunk and head, lanes for the tokens i: scores and dy v' into tensor memory beside S_0 dy; M's row sums from both; dy v' with its decays goes
// back in 16 bits and is multiplied with the keys.
template <typename T, int DK, int DV> __device__ __forceinline__ void grad_q(const GradDev& g)
{
    using S = GradShape<DK, DV>;
    const AttnDev& p = g.f;
    __shared__ Control ctl;
    __shared__ Decays dec;
    __shared__ alignas(16) float s_to[4][96];
    __shared__ float s_half[kChunk], s_rows[kChunk], s_within[kChunk], s_pairs[4][4], s_dot[8];
    const long long ci = blockIdx.x, at = ci * p.heads + blockIdx.y;
    const int head = blockIdx.y, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, quarter = warp % 4, half = warp / 4;
    wait_for_previous();
    const Chunk c = chunk_at(p, ci);
    if (c.len <= 0)
        return;
    char* smem = aligned_smem();
    const uint32_t queries = smem_u32(smem), keys = queries + S::K_BYTES, values = keys + S::K_BYTES, dys = values + S::V_BYTES, image = dys + S::V_BYTES;
    load_tile<T, DK, kThreads>(queries, p.q, c, head / p.share * p.dk, p.dk, p.vec_q, threadIdx.x);
    load_tile<T, DK, kThreads>(keys, p.k, c, head / p.share * p.dk, p.dk, p.vec_k, threadIdx.x);
    load_tile<T, DV, kThreads>(values, p.v, c, head * p.dv, p.dv, p.vec_v, threadIdx.x);
    load_tile<T, DV, kThreads>(dys, g.dy, c, head * p.dv, p.dv, g.vec_dy, threadIdx.x);
    load_image(image, g.image_S + at * (2 * S::IMAGE), 2 * S::IMAGE);
    copies_begun();
    // for <Z, S_0>: the image of Z comes into registers beside the tiles' copies
    constexpr int VECTORS = S::IMAGE / 16 / kThreads;
    uint4 other[2][VECTORS];
    if (g.want_l) {
        const uint4* from = reinterpret_cast<const uint4*>(g.image_Z + at * (2 * S::IMAGE)) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) {
            other[0][i] = from[i * kThreads];
            other[1][i] = from[S::IMAGE / 16 + i * kThreads];
        }
    }
    if (warp < 4)
        block_decays(log_decay_at<T>(p, c, head, threadIdx.x), threadIdx.x, dec);
    const uint32_t tmem = set_up(ctl, 512);      // scores, dy v', results: 128 columns each
    const uint32_t scores = tmem, slopes = tmem + 128, results = tmem + 256, lanes = (uint32_t)(quarter * 32) << 16;
    for (int i = threadIdx.x; i < 4 * 96; i += kThreads)
        s_to[i / 96][i % 96] = i % 96 < i / 96 * 32 ? to_block(dec, i % 96, i / 96) : 0.f;
    copies_done<0>();
    to_tensor_cores();
    __syncthreads();
    if (warp == 0) {
        constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, 128), id_state = instruction(kIsBf16<T>, false, false, 128, DK);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < DV / 16; ++s)
                mma(slopes, over_columns(dys, s), over_columns(values, s), id, s > 0);
#pragma unroll
            for (int s = 0; s < DK / 16; ++s)
                mma(scores, over_columns(queries, s), over_columns(keys, s), id, s > 0);
            commit(smem_u32(&ctl.bar[0]));
#pragma unroll
            for (int s = 0; s < DV / 16; ++s)
                mma(results, over_columns(dys, s), image_over_dv<DK>(image, s), id_state, s > 0);
#pragma unroll
            for (int s = 0; s < DV / 16; ++s)
                mma(results, over_columns(dys, s), image_over_dv<DK>(image + S::IMAGE, s), id_state, 1);
            commit(smem_u32(&ctl.bar[1]));
        }
        __syncwarp();
    }
    if (g.want_l) {                              // <Z, S_0>, while the products run
        const uint4* have = reinterpret_cast<const uint4*>(smem + 2 * S::K_BYTES + 2 * S::V_BYTES) + threadIdx.x;
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) {
            const uint4 x = have[i * kThreads], y = have[S::IMAGE / 16 + i * kThreads];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 a = unpack16<T>((&other[0][i].x)[j]), b = unpack16<T>((&other[1][i].x)[j]), c = unpack16<T>((&x.x)[j]), d = unpack16<T>((&y.x)[j]);
                dot = fmaf(a.x + b.x, c.x + d.x, dot);
                dot = fmaf(a.y + b.y, c.y + d.y, dot);
            }
        }
#pragma unroll
        for (int o = 16; o; o /= 2)
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
        if (lane == 0)
            s_dot[warp] = dot;
    }
    products_done(ctl, 0);
    const int row = quarter * 32 + lane;
    const float mine = dec.g[row], e_mine = ex2(mine);
    uint32_t packed[2][16];
    float row_sum = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int b = half + 2 * i;
        if (b <= quarter) {
            float v[32];
            tmem_ld32(slopes + b * 32 + lanes, v);
            decay_row(v, dec.g + b * 32, b == quarter, lane, mine, e_mine, &s_to[quarter][b < quarter ? b * 32 : 0]);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                packed[i][j] = pack16<T>(v[2 * j], v[2 * j + 1]);
            if (g.want_l) {
                float w[32];
                tmem_ld32(scores + b * 32 + lanes, w);
                if (b < quarter) {
                    float part = 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        part = fmaf(v[j], w[j], part);
                    row_sum += part;
#pragma unroll
                    for (int o = 16; o; o /= 2)
                        part += __shfl_xor_sync(0xffffffffu, part, o);
                    if (lane == 0)
                        s_pairs[quarter][b] = part;
                } else {
                    float x[32], sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        x[j] = j <= lane ? sum : 0.f;
                        sum = fmaf(v[j], w[j], sum);
                    }
                    group_sums<32, 32, 1>(x, lane);
                    s_within[b * 32 + first_value<32, 32>(lane)] = x[0];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                packed[i][j] = 0;
        }
    }
    before_barrier();
    asm volatile("bar.sync %0, 64;" :: "r"(1 + quarter) : "memory");
    behind_barrier();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        tmem_st16(slopes + (half + 2 * i) * 16 + lanes, packed[i]);
    products_done(ctl, 1);
    const float e = weigh_row<T, DK>(results + lanes, smem, row, half, from_begin(dec, row) * (kIsBf16<T> ? 1.f : g.unit_S[at]));
    if (half == 1) {
        s_half[row] = e;
        s_rows[row] = row_sum;
    }
    tmem_st_done();
    before_barrier();
    __syncthreads();
    if (warp == 0) {
        behind_barrier();
        constexpr uint32_t id = instruction(kIsBf16<T>, false, true, 128, DK);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < 8; ++s)
                mma_tmem(results, slopes + s * 8, over_tokens(keys, s), id, 1);
            commit(smem_u32(&ctl.bar[2]));
        }
        __syncwarp();
    }
    if (half == 0 && g.want_l) {
        const long long plane = (long long)p.heads * p.chunks * kChunk;
        float* to = g.tokens + ((long long)head * p.chunks + ci) * kChunk + row;
        to[0] = (e + s_half[row]) * p.scale;
        to[plane] = (row_sum + s_rows[row]) * p.scale;
        to[4 * plane] = s_within[row] * p.scale;
        if (row == 0) {
            float dot = 0.f;
            for (int i = 0; i < 8; ++i)
                dot += s_dot[i];
            g.across[at] = dot * over_chunk(dec) * (kIsBf16<T> ? 1.f : g.unit_S[at] * g.unit_Z[at]);
        }
        if (row < 2)
            g.bridges[2 * at + row] = (s_pairs[3][0] + s_pairs[2 + row][row]) * p.scale;
    }
    products_done(ctl, 2);
    if (g.part_q)
        part_row<DK>(results + lanes, g.part_q + (packed_row(p, c, row) * p.heads + head) * p.dk, p.dk, row < c.len, half, p.scale);
    else if (g.dq.ptr)
        stage_row<T, DK>(results + lanes, smem, row, half, p.scale);
    give_back(tmem, 512);
    if (!g.part_q && g.dq.ptr)
        store_tile<T, DK>(smem, g.dq, c, head, p.dk, g.vec_dq);
}

// Decay of the pairs (32 rows of block b, column) of the lower triangle, a lane for the column j: `mine` its sum from its block's begin, `to_there` the decay from it
// to block b's begin; from [32]: the rows' decays from there.
__device__ __forceinline__ void decay_column(float (&v)[32], const Decays& d, bool diagonal, int b, int lane, float mine, float to_there, const float* from)
{
    if (diagonal) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const float4 h = *reinterpret_cast<const float4*>(d.g + b * 32 + i);
            v[i] = i >= lane ? v[i] * ex2(h.x - mine) : 0.f;
            v[i + 1] = i + 1 >= lane ? v[i + 1] * ex2(h.y - mine) : 0.f;
            v[i + 2] = i + 2 >= lane ? v[i + 2] * ex2(h.z - mine) : 0.f;
            v[i + 3] = i + 3 >= lane ? v[i + 3] * ex2(h.w - mine) : 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const float4 h = *reinterpret_cast<const float4*>(from + i);
            v[i] *= to_there * h.x;
            v[i + 1] *= to_there * h.y;
            v[i + 2] *= to_there * h.z;
            v[i + 3] *= to_there * h.w;
        }
    }
}

// dk and dv of one chunk and head, lanes for the tokens j.
template <typename T, int DK, int DV> __device__ __forceinline__ void grad_kv(const GradDev& g)
{
    using S = GradShape<DK, DV>;
    const AttnDev& p = g.f;
    __shared__ Control ctl;
    __shared__ Decays dec;
    __shared__ alignas(16) float s_from[kChunk];
    __shared__ float s_f[kChunk], s_col[kChunk];
    const long long ci = blockIdx.x, at = ci * p.heads + blockIdx.y;
    const int head = blockIdx.y, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, quarter = warp % 4, half = warp / 4;
    wait_for_previous();
    const Chunk c = chunk_at(p, ci);
    if (c.len <= 0)
        return;
    char* smem = aligned_smem();
    const uint32_t queries = smem_u32(smem), keys = queries + S::K_BYTES, values = keys + S::K_BYTES, dys = values + S::V_BYTES, image = dys + S::V_BYTES;
    char* s_keys = smem + S::K_BYTES;
    char* s_values = s_keys + S::K_BYTES;
    load_tile<T, DK, kThreads>(queries, p.q, c, head / p.share * p.dk, p.dk, p.vec_q, threadIdx.x);
    load_tile<T, DK, kThreads>(keys, p.k, c, head / p.share * p.dk, p.dk, p.vec_k, threadIdx.x);
    load_tile<T, DV, kThreads>(values, p.v, c, head * p.dv, p.dv, p.vec_v, threadIdx.x);
    load_tile<T, DV, kThreads>(dys, g.dy, c, head * p.dv, p.dv, g.vec_dy, threadIdx.x);
    load_image(image, g.image_Z + at * (2 * S::IMAGE), 2 * S::IMAGE);
    copies_begun();
    if (warp < 4)
        block_decays(log_decay_at<T>(p, c, head, threadIdx.x), threadIdx.x, dec);
    const uint32_t tmem = set_up(ctl, 512);      // scores, v dy', dk, dv: 128 columns each
    const uint32_t scores = tmem, slopes = tmem + 128, dks = tmem + 256, dvs = tmem + 384, lanes = (uint32_t)(quarter * 32) << 16;
    if (warp < 4)
        s_from[threadIdx.x] = ex2(dec.g[threadIdx.x]);
    copies_done<0>();
    to_tensor_cores();
    __syncthreads();
    if (warp == 0) {
        constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, 128), id_k = instruction(kIsBf16<T>, false, false, 128, DK),
                           id_v = instruction(kIsBf16<T>, false, true, 128, DV);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < DV / 16; ++s)
                mma(slopes, over_columns(values, s), over_columns(dys, s), id, s > 0);
#pragma unroll
            for (int s = 0; s < DK / 16; ++s)
                mma(scores, over_columns(keys, s), over_columns(queries, s), id, s > 0);
            commit(smem_u32(&ctl.bar[0]));
#pragma unroll
            for (int s = 0; s < DV / 16; ++s)
                mma(dks, over_columns(values, s), image_over_dv<DK>(image, s), id_k, s > 0);
#pragma unroll
            for (int s = 0; s < DV / 16; ++s)
                mma(dks, over_columns(values, s), image_over_dv<DK>(image + S::IMAGE, s), id_k, 1);
#pragma unroll
            for (int s = 0; s < DK / 16; ++s)
                mma(dvs, over_columns(keys, s), image_over_dk<DK>(image, s), id_v, s > 0);
            commit(smem_u32(&ctl.bar[1]));
        }
        __syncwarp();
    }
    products_done(ctl, 0);
    const int row = quarter * 32 + lane;
    const float mine = dec.g[row];
    uint32_t packed_v[2][16], packed_k[2][16];
    float col = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int b = half + 2 * i;
        if (b >= quarter) {
            const float to_there = b > quarter ? to_block(dec, row, b) * p.scale : 0.f;
            float v[32], w[32];
            tmem_ld32(scores + b * 32 + lanes, v);
            tmem_ld32(slopes + b * 32 + lanes, w);
            // M = decay scale (q . k) (dy . v): the decay goes into the scores first, then into the slopes
            decay_column(v, dec, b == quarter, b, lane, mine, to_there, s_from + b * 32);
            if (b == quarter) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    v[j] *= p.scale;
            }
            if (b > quarter) {
                float part = 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    part = fmaf(v[j], w[j], part);
                col += part;
            }
            decay_column(w, dec, b == quarter, b, lane, mine, to_there, s_from + b * 32);
            if (b == quarter) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    w[j] *= p.scale;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                packed_v[i][j] = pack16<T>(v[2 * j], v[2 * j + 1]);
                packed_k[i][j] = pack16<T>(w[2 * j], w[2 * j + 1]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                packed_v[i][j] = packed_k[i][j] = 0;
        }
    }
    before_barrier();
    asm volatile("bar.sync %0, 64;" :: "r"(1 + quarter) : "memory");
    behind_barrier();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        tmem_st16(scores + (half + 2 * i) * 16 + lanes, packed_v[i]);
        tmem_st16(slopes + (half + 2 * i) * 16 + lanes, packed_k[i]);
    }
    products_done(ctl, 1);
    const float f = to_end(dec, row) * (kIsBf16<T> ? 1.f : g.unit_Z[at]);
    const float fj = weigh_row<T, DK>(dks + lanes, s_keys, row, half, f);
    weigh_row<T, DV>(dvs + lanes, nullptr, row, half, f);
    if (half == 1) {
        s_f[row] = fj;
        s_col[row] = col;
    }
    tmem_st_done();
    before_barrier();
    __syncthreads();
    if (warp == 0) {
        behind_barrier();
        constexpr uint32_t id_k = instruction(kIsBf16<T>, false, true, 128, DK), id_v = instruction(kIsBf16<T>, false, true, 128, DV);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < 8; ++s)
                mma_tmem(dvs, scores + s * 8, over_tokens(dys, s), id_v, 1);
#pragma unroll
            for (int s = 0; s < 8; ++s)
                mma_tmem(dks, slopes + s * 8, over_tokens(queries, s), id_k, 1);
            commit(smem_u32(&ctl.bar[2]));
        }
        __syncwarp();
    }
    if (half == 0 && g.want_l) {
        const long long plane = (long long)p.heads * p.chunks * kChunk;
        float* to = g.tokens + ((long long)head * p.chunks + ci) * kChunk + row;
        to[2 * plane] = fj + s_f[row];
        to[3 * plane] = col + s_col[row];
    }
    products_done(ctl, 2);
    if (g.part_k)
        part_row<DK>(dks + lanes, g.part_k + (packed_row(p, c, row) * p.heads + head) * p.dk, p.dk, row < c.len, half, 1.f);
    else if (g.dk.ptr)
        stage_row<T, DK>(dks + lanes, s_keys, row, half, 1.f);
    if (g.dv.ptr)
        stage_row<T, DV>(dvs + lanes, s_values, row, half, 1.f);
    give_back(tmem, 512);
    if (!g.part_k && g.dk.ptr)
        store_tile<T, DK>(s_keys, g.dk, c, head, p.dk, g.vec_dk);
    if (g.dv.ptr)
        store_tile<T, DV>(s_values, g.dv, c, head, p.dv, g.vec_dv);
}

// Both in one launch (blockIdx.z), whose last round of blocks is then half as long.
template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads, 1) grad_kernel(const GradDev g)
{
    if (blockIdx.z == 0 && g.want_kv)
        grad_kv<T, DK, DV>(g);
    else
        grad_q<T, DK, DV>(g);
}

// Sums of dq and dk over the heads of a group, one block per token row, in the order of the heads.
template <typename T>
__global__ void __launch_bounds__(kThreads) grad_group_kernel(const GradDev g)
{
    wait_for_previous();
    const AttnDev& p = g.f;
    const Chunk c = chunk_at(p, blockIdx.x);
    const int n = p.heads / p.share * p.dk;
    for (int t = blockIdx.y; t < c.len; t += gridDim.y) {
        const long long row = packed_row(p, c, t) * p.heads * p.dk;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const long long from = row + (long long)(i / p.dk) * p.share * p.dk + i % p.dk;
            float q = 0.f, k = 0.f;
            for (int h = 0; h < p.share; ++h) {
                if (g.part_q)
                    q += g.part_q[from + (long long)h * p.dk];
                if (g.part_k)
                    k += g.part_k[from + (long long)h * p.dk];
            }
            if (g.part_q)
                row_ptr<T>(g.dq, c.seq, c.row0 + t)[i] = from_f<T>(q);
            if (g.part_k)
                row_ptr<T>(g.dk, c.seq, c.row0 + t)[i] = from_f<T>(k);
        }
    }
}

// dl of one chunk and head, one warp, four tokens to a lane; what follows from it for delta, and the chunk's shares of dA and ddelta_bias.
template <typename T>
__global__ void __launch_bounds__(128) grad_decay_kernel(const GradDev g)
{
    wait_for_previous();
    const AttnDev& p = g.f;
    const int lane = threadIdx.x % 32;
    const long long ci = blockIdx.x;
    const int head = blockIdx.y * 4 + threadIdx.x / 32;
    if (head >= p.heads)
        return;
    const Chunk c = chunk_at(p, ci);
    const long long plane = (long long)p.heads * p.chunks * kChunk, at = ((long long)head * p.chunks + ci) * kChunk + lane * 4;
    float sum_A = 0.f, sum_bias = 0.f;
    if (c.len > 0) {
        float e[4], rows[4], f[4], cols[4], dl[4];
        auto load = [&](int i, float (&v)[4]) {
            const float4 x = *reinterpret_cast<const float4*>(g.tokens + i * plane + at);
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        };
        load(0, e), load(1, rows), load(2, f), load(3, cols), load(4, dl);
        // from t on: e over the chunk, row sums over the block of 8 lanes; in front of t: f over the chunk, column sums over the block
        auto four = [](const float (&v)[4]) { return (v[0] + v[1]) + (v[2] + v[3]); };
        float sum_e = four(e), sum_rows = four(rows), sum_f = four(f), sum_cols = four(cols);
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const float x = __shfl_down_sync(0xffffffffu, sum_e, o), y = __shfl_up_sync(0xffffffffu, sum_f, o);
            sum_e += lane + o < 32 ? x : 0.f;
            sum_f += lane >= o ? y : 0.f;
        }
#pragma unroll
        for (int o = 1; o < 8; o *= 2) {
            const float x = __shfl_down_sync(0xffffffffu, sum_rows, o, 8), y = __shfl_up_sync(0xffffffffu, sum_cols, o, 8);
            sum_rows += lane % 8 + o < 8 ? x : 0.f;
            sum_cols += lane % 8 >= o ? y : 0.f;
        }
        // of the other lanes
        const float x = __shfl_down_sync(0xffffffffu, sum_e, 1), y = __shfl_up_sync(0xffffffffu, sum_f, 1);
        const float z = __shfl_down_sync(0xffffffffu, sum_rows, 1, 8), w = __shfl_up_sync(0xffffffffu, sum_cols, 1, 8);
        float behind = (lane < 31 ? x : 0.f) + (lane % 8 < 7 ? z : 0.f), front = (lane ? y : 0.f) + (lane % 8 ? w : 0.f);
        const int block = lane / 8;
        const long long ch = ci * p.heads + head;
        const float over = g.across[ch] + (block == 1 || block == 2 ? g.bridges[2 * ch + block - 1] : 0.f);
        const float A = p.A[head];
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            behind += e[i] + rows[i];
            dl[i] += behind;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dl[i] += front + over;
            front += f[i] + cols[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = lane * 4 + i;
            if (t >= c.len)
                continue;
            float step = 1.f, slope = 1.f;
            if (p.delta.ptr) {
                const float raw = raw_step<T>(p, c.seq, c.row0 + t, head);
                step = step_of(p, raw);
                slope = p.softplus ? sigmoid(raw) : 1.f;
            }
            const float d = dl[i] * A * slope;
            sum_A = fmaf(dl[i], step, sum_A);
            sum_bias += d;
            if (g.ddelta.ptr)
                row_ptr<T>(g.ddelta, c.seq, c.row0 + t)[head] = from_f<T>(d);
        }
    }
#pragma unroll
    for (int o = 16; o; o /= 2) {
        sum_A += __shfl_xor_sync(0xffffffffu, sum_A, o);
        sum_bias += __shfl_xor_sync(0xffffffffu, sum_bias, o);
    }
    if (lane == 0) {
        g.sums[(long long)head * p.chunks + ci] = sum_A;
        g.sums[((long long)p.heads + head) * p.chunks + ci] = sum_bias;
    }
}

// Sums over the chunks, one block to each head and sum.
static __global__ void __launch_bounds__(kThreads) grad_head_kernel(const GradDev g)
{
    wait_for_previous();
    __shared__ float s_sum[8];
    const AttnDev& p = g.f;
    float* to = blockIdx.y ? g.dbias : g.dA;
    if (!to)
        return;
    const float* from = g.sums + ((long long)blockIdx.y * p.heads + blockIdx.x) * p.chunks;
    float sum = 0.f;
    for (long long i = threadIdx.x; i < p.chunks; i += kThreads)
        sum += from[i];
#pragma unroll
    for (int o = 16; o; o /= 2)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x % 32 == 0)
        s_sum[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.f;
        for (int i = 0; i < 8; ++i)
            sum += s_sum[i];
        to[blockIdx.x] = sum;
    }
}

} // namespace dattn
} // namespace ttc
