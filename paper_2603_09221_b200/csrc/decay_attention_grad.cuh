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
// dl goes into float32 sums over all tokens (dA, ddelta_bias): M is taken from the float32 scores, and S_0 and Z go into e and f as sums of numbers of 16 bits, three
// bfloat16 (2^-27 of the value; with two, 2^-18, dA was off by up to 7e-6 of its norm) or two float16 (2^-23).  dq, dk and dv alone make do with two.
//
// The states in front of the chunks come from a state walk, the Z from one that goes backwards along queries and dy; then one
// kernel finds dq, e and row, one dk, dv, f and col, and a small one dl.
#pragma once

#include "decay_attention.cuh"

namespace ttc {
namespace dattn {

struct GradDev {
    AttnDev f;
    Rows dy, dq, dk, dv, ddelta;
    int head_dy;                                 // as f.head_v
    int vec_dq, vec_dk, vec_dv;
    const float* dstate_out;
    float *dA, *dbias, *dstate;
    // scratch
    float *part_q, *part_k;                      // dq, dk of every head, where heads share them: [rows][heads][dk]
    char *image_S, *image_Z;                     // [chunks][heads][terms][DV / 8][DK][8]
    int terms;
    float *unit_S, *unit_Z;
    float* tokens;                               // [5][heads][chunks][128]: e, row sums, f, column sums (both without the blocks on the diagonal), pairs within t's block
    float* bridges;                              // [chunks][heads][2]: of pairs on both sides of the second and the third block
    float* across;                               // exp(G_C) <Z, S_0>: shares, [chunks][heads][across_of]
    int across_of;
    float* whole;                                // exp(G_C), [chunks][heads], where <Z, S_0> has a kernel of its own
    float* sums;                                 // of dA and of ddelta_bias: [2][heads][chunks]
    int want_q, want_kv, want_l;
    int resident;                                // blocks that run at once
};

constexpr int kGradThreads = 512;

template <int DK, int DV> struct GradShape {
    static constexpr int K_BYTES = DK / 64 * kBox, V_BYTES = DV / 64 * kBox, IMAGE = DK * DV * 2;
    static constexpr int TILES = 2 * K_BYTES + 2 * V_BYTES + 2 * IMAGE;
    struct Small {
        Control ctl;
        uint64_t tiles, image;                                       // what has come: the tiles, two terms of the image
        uint64_t second_product, third, third_product;               // of the images' terms: products that are done, the third term is there
        Decays dec;
        alignas(16) float to[4][96];             // [block][earlier token]: decay from it to the block's begin
        alignas(16) float from[kChunk];          // exp from each token's block's begin
        float sums[4][kChunk], dots[4][kChunk], within[4][kChunk], pairs[4][4];
        float most[2][4][kChunk];                // float16: the largest weights of a row's warps
    };
    static constexpr int SMEM = TILES + sizeof(Small);
};

// A quarter of a row of results (COLS / 4 of tensor memory's columns), times f, staged in a tile.
template <typename T, int COLS> __device__ __forceinline__ void stage_row(uint32_t from, char* tile, int row, int sub, float f)
{
#pragma unroll 1
    for (int c0 = 0; c0 < COLS / 4; c0 += 16) {
        float v[16];
        tmem_ld16(from + sub * (COLS / 4) + c0, v);
#pragma unroll
        for (int j = 0; j < 16; j += 8) {
            const uint4 w = make_uint4(pack16<T>(v[j] * f, v[j + 1] * f), pack16<T>(v[j + 2] * f, v[j + 3] * f), pack16<T>(v[j + 4] * f, v[j + 5] * f),
                                       pack16<T>(v[j + 6] * f, v[j + 7] * f));
            *reinterpret_cast<uint4*>(tile + tile_at(row, (sub * (COLS / 4) + c0 + j) / 8)) = w;
        }
    }
}
// The same in float32, [128][COLS], 16 bytes in another place of their 128 in each of eight rows.
template <int COLS> __device__ __forceinline__ float4* part_at(char* area, int row, int c4) { return reinterpret_cast<float4*>(area) + row * (COLS / 4) + (c4 ^ (row & 7)); }
template <int COLS> __device__ __forceinline__ void stage_part(uint32_t from, char* area, int row, int sub, float f)
{
#pragma unroll 1
    for (int c0 = 0; c0 < COLS / 4; c0 += 16) {
        float v[16];
        tmem_ld16(from + sub * (COLS / 4) + c0, v);
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            *part_at<COLS>(area, row, (sub * (COLS / 4) + c0 + j) / 4) = make_float4(v[j] * f, v[j + 1] * f, v[j + 2] * f, v[j + 3] * f);
    }
}
// From there to a head's part of a sum over the heads of a group.
template <int COLS> __device__ __forceinline__ void store_part(char* area, float* to, long long stride, int rows, int width)
{
    for (int e = threadIdx.x; e < kChunk * COLS / 4; e += kGradThreads) {
        const int row = e / (COLS / 4), c4 = e % (COLS / 4);
        if (row >= rows || c4 * 4 >= width)
            continue;
        const float4 v = *part_at<COLS>(area, row, c4);
        float* at = to + row * stride + c4 * 4;
        if (width % 4 == 0) {
            *reinterpret_cast<float4*>(at) = v;
        } else {
            at[0] = v.x;
            if (c4 * 4 + 1 < width)
                at[1] = v.y;
            if (c4 * 4 + 2 < width)
                at[2] = v.z;
            if (c4 * 4 + 3 < width)
                at[3] = v.w;
        }
    }
}
// A quarter of a row of results, times f, back to where it was; returns its product with the same quarter of row `row` of a tile.
template <typename T, int COLS> __device__ __forceinline__ float weigh_row(uint32_t at, const char* tile, int row, int sub, float f)
{
    float dot = 0.f;
#pragma unroll 1
    for (int c0 = 0; c0 < COLS / 4; c0 += 16) {
        float v[16];
        const uint32_t here = at + sub * (COLS / 4) + c0;
        tmem_ld16(here, v);
        uint32_t r[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            v[j] *= f;
            r[j] = __float_as_uint(v[j]);
        }
        if (tile) {
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
                const uint4 w = *reinterpret_cast<const uint4*>(tile + tile_at(row, (sub * (COLS / 4) + c0 + j) / 8));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 x = unpack16<T>((&w.x)[i]);
                    dot = fmaf(x.x, v[j + 2 * i], dot);
                    dot = fmaf(x.y, v[j + 2 * i + 1], dot);
                }
            }
        }
        tmem_st16(here, r);
    }
    return dot;
}

// float16: the power of two that a row's weights are taken times, from what its four warps have left in `most`; `inverse` of it.
__device__ __forceinline__ float power_of_row(const float (&most)[4][kChunk], int row, float unit, float& inverse)
{
    return row_power(fmaxf(fmaxf(most[0][row], most[1][row]), fmaxf(most[2][row], most[3][row])), highest_with(unit), inverse);
}

__device__ __forceinline__ long long packed_row(const AttnDev& p, const Chunk& c, int t) { return c.seq * p.seqs.tokens + c.row0 + t; }

__device__ __forceinline__ void fetch_bytes(uint32_t to, const char* from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" :: "r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void fetch_bytes_to_l2(const char* from, uint32_t bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" :: "l"(from), "r"(bytes) : "memory");
}

// Chunk and head of a block: those of one head one behind the other, both ways (dk and dv, dq) of a chunk together.
struct GradPlace {
    int chunk, head;
    bool kv;
};
__device__ __forceinline__ GradPlace grad_place(const GradDev& g, unsigned id)
{
    const unsigned ways = g.want_q && g.want_kv ? 2 : 1, job = id / ways, chunks = (unsigned)g.f.chunks;
    return GradPlace{(int)(job % chunks), (int)(job / chunks), g.want_kv && (ways == 1 || id % 2 == 0)};
}

// The tiles of a chunk and head and its decays; its image is asked for.  The copies are under way before tensor memory is taken.
template <typename T, int DK, int DV, bool KV>
__device__ __forceinline__ uint32_t begin_grad(const GradDev& g, const Maps& there, const Maps& back, const Chunk& c, long long at, int head, typename GradShape<DK, DV>::Small& sm,
                                               uint32_t tiles)
{
    using S = GradShape<DK, DV>;
    const AttnDev& p = g.f;
    const int group = head / p.share, warp = threadIdx.x / 32;
    const uint32_t queries = tiles, keys = queries + S::K_BYTES, values = keys + S::K_BYTES, dys = values + S::V_BYTES, image = dys + S::V_BYTES;
    const bool engine = !p.seqs.offsets || c.len == kChunk;
    const uint32_t bar = smem_u32(&sm.tiles);
    if (threadIdx.x == kGradThreads - 32) {
        for (uint64_t* b : {&sm.tiles, &sm.image, &sm.second_product, &sm.third, &sm.third_product})
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(smem_u32(b)) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        expect_bytes(bar, engine ? 2 * S::K_BYTES + 2 * S::V_BYTES : 0);
        if (engine) {
            const int row0 = (int)c.row0, seq = (int)c.seq;
            for (int b = 0; b < DV / 64; ++b) {
                fetch_box(values + b * kBox, &there.v, b * 64, head, row0, seq, bar);
                fetch_box(dys + b * kBox, &back.v, b * 64, head, row0, seq, bar);
            }
            for (int b = 0; b < DK / 64; ++b) {
                fetch_box(keys + b * kBox, &there.k, b * 64, group, row0, seq, bar);
                fetch_box(queries + b * kBox, &back.k, b * 64, group, row0, seq, bar);
            }
        }
        expect_bytes(smem_u32(&sm.image), 2 * S::IMAGE);
        fetch_bytes(image, (KV ? g.image_Z : g.image_S) + at * ((long long)g.terms * S::IMAGE), 2 * S::IMAGE, smem_u32(&sm.image));
    }
    float l = 0.f;
    if (warp < 4)
        l = log_decay_at<T>(p, c, head, threadIdx.x);
    const uint32_t tmem = set_up(sm.ctl, 512);
    if (!engine) {
        load_tile<T, DK, kGradThreads>(queries, p.q, c, group * p.head_q, p.dk, threadIdx.x);
        load_tile<T, DK, kGradThreads>(keys, p.k, c, group * p.head_k, p.dk, threadIdx.x);
        load_tile<T, DV, kGradThreads>(values, p.v, c, head * p.head_v, p.dv, threadIdx.x);
        load_tile<T, DV, kGradThreads>(dys, g.dy, c, head * g.head_dy, p.dv, threadIdx.x);
        copies_begun();
    }
    if (warp < 4) {
        block_decays(l, threadIdx.x, sm.dec);
        sm.from[threadIdx.x] = ex2(sm.dec.g[threadIdx.x]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * 96; i += kGradThreads)
        sm.to[i / 96][i % 96] = i % 96 < i / 96 * 32 ? to_block(sm.dec, i % 96, i / 96) : 0.f;
    copies_done<0>();
    await(bar, 0, &sm.ctl.dead);
    to_tensor_cores();
    __syncthreads();
    behind_barrier();
    return tmem;
}
// What the block that will run behind this one needs is asked for into L2, so that memory is at work while this one computes.  By a thread that has nothing else to do.
template <int DK, int DV> __device__ __forceinline__ void fetch_next(const GradDev& g, const Maps& there, const Maps& back)
{
    const AttnDev& p = g.f;
    const unsigned next = blockIdx.x + g.resident;
    if (next >= gridDim.x)
        return;
    const GradPlace where = grad_place(g, next);
    const Chunk n = chunk_at(p, where.chunk);
    if (n.len <= 0)
        return;
    const int row0 = (int)n.row0, seq = (int)n.seq, group = where.head / p.share;
    for (int b = 0; b < DV / 64; ++b) {
        fetch_to_l2(&there.v, b * 64, where.head, row0, seq);
        fetch_to_l2(&back.v, b * 64, where.head, row0, seq);
    }
    for (int b = 0; b < DK / 64; ++b) {
        fetch_to_l2(&there.k, b * 64, group, row0, seq);
        fetch_to_l2(&back.k, b * 64, group, row0, seq);
    }
    const int bytes = g.terms * GradShape<DK, DV>::IMAGE;
    fetch_bytes_to_l2((where.kv ? g.image_Z : g.image_S) + ((long long)where.chunk * p.heads + where.head) * bytes, bytes);
}
__device__ __forceinline__ void grad_products_done(Control& c, int i)
{
    await(smem_u32(&c.bar[i]), 0, &c.dead);
    __syncwarp();
    behind_barrier();
}
// (products under way end before tensor memory is given back)
__device__ __forceinline__ void end_grad(Control& c, uint32_t tmem)
{
    before_barrier();
    __syncthreads();
    if (threadIdx.x / 32 == 4) {
        if (c.dead) {
            if (threadIdx.x % 32 == 0)
                for (int i = 0; i < 1000; ++i)
                    __nanosleep(1000);
            __syncwarp();
        }
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512) : "memory");
    }
}

// dq of one chunk and head, lanes for the tokens i, a block of 32 tokens j to each of a row's four warps: scores and dy v' into tensor memory beside S_0 dy; M's row sums from both;
// dy v' with its decays goes back in 16 bits and is multiplied with the keys.
template <typename T, int DK, int DV> __device__ __forceinline__ void grad_q(const GradDev& g, const Maps& there, const Maps& back, const GradPlace& where)
{
    using S = GradShape<DK, DV>;
    const AttnDev& p = g.f;
    const long long ci = where.chunk, at = ci * p.heads + where.head;
    const int head = where.head;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, quarter = warp % 4, sub = warp / 4;
    const Chunk c = chunk_at(p, ci);
    if (c.len <= 0)
        return;
    char* smem = dattn_tiles;
    typename S::Small& sm = *reinterpret_cast<typename S::Small*>(smem + S::TILES);
    const Decays& dec = sm.dec;
    const uint32_t queries = __shfl_sync(0xffffffffu, smem_u32(smem), 0), keys = queries + S::K_BYTES, values = keys + S::K_BYTES, dys = values + S::V_BYTES,
                   image = dys + S::V_BYTES;
    const uint32_t tmem = begin_grad<T, DK, DV, false>(g, there, back, c, at, head, sm, queries);        // scores, dy v', results: 128 columns each
    const uint32_t scores = tmem, slopes = tmem + 128, results = tmem + 256, lanes = (uint32_t)(quarter * 32) << 16;
    if (warp == 0) {
        constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, 128);
        if (elect_one()) {
            products<DV / 16, kColumns, kColumns>(slopes, over_columns(dys, 0), over_columns(values, 0), id, false);
            products<DK / 16, kColumns, kColumns>(scores, over_columns(queries, 0), over_columns(keys, 0), id, false);
            commit(smem_u32(&sm.ctl.bar[0]));
        }
        __syncwarp();
    }
    if (warp == 12) {                            // (of the first 32 rows' warps, which have the fewest pairs to weigh, as warp 8)
        constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, DK);
        await(smem_u32(&sm.image), 0, &sm.ctl.dead);
        __syncwarp();
        if (elect_one()) {
            products<DV / 16, kColumns, 2 * DK>(results, over_columns(dys, 0), image_over_dv<DK>(image + S::IMAGE, 0), id, false); // the small ones first: the tensor cores cut sums off
            products<DV / 16, kColumns, 2 * DK>(results, over_columns(dys, 0), image_over_dv<DK>(image, 0), id, true);
            commit(smem_u32(&sm.ctl.bar[1]));
        }
        __syncwarp();
    } else if (warp == 8) {
        if (elect_one())
            fetch_next<DK, DV>(g, there, back);
        __syncwarp();
    }
    grad_products_done(sm.ctl, 0);
    if (g.terms == 3 && warp == 12) {            // the third term takes the values' place
        if (elect_one()) {
            expect_bytes(smem_u32(&sm.third), S::IMAGE);
            fetch_bytes(values, g.image_S + (at * 3 + 2) * S::IMAGE, S::IMAGE, smem_u32(&sm.third));
        }
        __syncwarp();
    }
    // A warp has one of the earlier blocks of 32 tokens and a quarter of its rows' own block, where the exponentials are (packed
    // documents, 8 heads of 64 x 64: 130.4 -> 129.3 us).
    const int row = quarter * 32 + lane;
    uint32_t packed[16], diagonal[4];
    float most = 0.f, most_own = 0.f, over = 0.f, over_own = 0.f;
    float row_sum = 0.f;
    if (sub < quarter) {
        float v[32];
        tmem_ld32(slopes + sub * 32 + lanes, v);
        decay_earlier(v, sm.from[row], sm.to[quarter] + sub * 32);
        pack_weights<T>(v, packed, most, over);
        if (g.want_l) {
            float w[32];
            tmem_ld32(scores + sub * 32 + lanes, w);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                row_sum = fmaf(v[j], w[j], row_sum);
            float part = row_sum;
#pragma unroll
            for (int o = 16; o; o /= 2)
                part += __shfl_xor_sync(0xffffffffu, part, o);
            if (lane == 0)
                sm.pairs[quarter][sub] = part;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            packed[j] = 0;
    }
    {
        const int first = sub * 8, from = quarter * 32 + first;
        const float own = dec.g[row], own_low = dec.low[row];
        float v[8];
        tmem_ld8(slopes + from + lanes, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = first + j <= lane ? v[j] * ex2((own - dec.g[from + j]) + (own_low - dec.low[from + j])) : 0.f;
        pack_weights<T>(v, diagonal, most_own, over_own);
        if (g.want_l) {                          // pairs on both sides of t whose earlier token is one of these eight: of t among them one by one, of a later t all
            float w[8], sum = 0.f;
            tmem_ld8(scores + from + lanes, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = v[j] * w[j];
                v[j] = first + j <= lane ? sum : 0.f;
                sum += m;
            }
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float b = __shfl_down_sync(0xffffffffu, sum, o);
                sum += lane + o < 32 ? b : 0.f;
            }
            group_sums<8, 32, 1>(v, lane);
            if (lane < first || lane >= first + 8)
                sm.within[sub][row] = lane < first ? 0.f : sum;
            if (lane < 8)
                sm.within[sub][from + first_value<8, 32>(lane)] = v[0];
        }
    }
    if (!kIsBf16<T>)
        sm.most[0][sub][row] = fmaxf(most, most_own);
    // the four warps of these rows have read what is overwritten now
    before_barrier();
    asm volatile("bar.sync %0, 128;" :: "r"(1 + quarter) : "memory");
    behind_barrier();
    float up = 1.f, down = 1.f;
    if (!kIsBf16<T>) {
        const float unit = g.unit_S[at];
        up = power_of_row(sm.most[0], row, unit, down);
        change_power(packed, up * over);
        change_power(diagonal, up * over_own);
        up *= unit;
    }
    if (sub != quarter)
        tmem_st16(slopes + sub * 16 + lanes, packed);
    tmem_st4(slopes + quarter * 16 + sub * 4 + lanes, diagonal);
    if (g.terms == 3 && warp == 12) {
        constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, DK);
        await(smem_u32(&sm.third), 0, &sm.ctl.dead);
        __syncwarp();
        if (elect_one()) {
            products<DV / 16, kColumns, 2 * DK>(results, over_columns(dys, 0), image_over_dv<DK>(values, 0), id, true);
            commit(smem_u32(&sm.third_product));
        }
        __syncwarp();
    }
    grad_products_done(sm.ctl, 1);
    if (g.terms == 3) {
        await(smem_u32(&sm.third_product), 0, &sm.ctl.dead);
        __syncwarp();
        behind_barrier();
    }
    sm.dots[sub][row] = weigh_row<T, DK>(results + lanes, smem, row, sub, from_begin(dec, row) * up) * down;
    sm.sums[sub][row] = row_sum;
    tmem_st_done();
    before_barrier();
    __syncthreads();
    if (warp == 0) {
        behind_barrier();
        constexpr uint32_t id = instruction(kIsBf16<T>, false, true, 128, DK);
        if (elect_one()) {
            products_tmem<8, kTokens>(results, slopes, over_tokens(keys, 0), id);
            commit(smem_u32(&sm.ctl.bar[2]));
        }
        __syncwarp();
    }
    if (sub == 0 && g.want_l) {
        const long long plane = (long long)p.heads * p.chunks * kChunk;
        float* to = g.tokens + ((long long)head * p.chunks + ci) * kChunk + row;
        to[0] = ((sm.dots[0][row] + sm.dots[1][row]) + (sm.dots[2][row] + sm.dots[3][row])) * p.scale;
        to[plane] = ((sm.sums[0][row] + sm.sums[1][row]) + (sm.sums[2][row] + sm.sums[3][row])) * p.scale;
        to[4 * plane] = ((sm.within[0][row] + sm.within[1][row]) + (sm.within[2][row] + sm.within[3][row])) * p.scale;
        if (row < 2)
            g.bridges[2 * at + row] = (sm.pairs[3][0] + sm.pairs[2 + row][row]) * p.scale;
    }
    grad_products_done(sm.ctl, 2);
    if (g.part_q)                                // (in the place of queries and keys)
        stage_part<DK>(results + lanes, smem, row, sub, p.scale * down);
    else if (g.dq.ptr)
        stage_row<T, DK>(results + lanes, smem, row, sub, p.scale * down);
    end_grad(sm.ctl, tmem);
    if (g.part_q)
        store_part<DK>(smem, g.part_q + (packed_row(p, c, 0) * p.heads + head) * p.dk, (long long)p.heads * p.dk, c.len, p.dk);
    else if (g.dq.ptr)
        store_tile<T, DK, kGradThreads>(smem, g.dq, c, head, p.dk, g.vec_dq);
}

// dk and dv of one chunk and head, lanes for the tokens j, a block of 32 tokens i to each of a row's four warps.
template <typename T, int DK, int DV> __device__ __forceinline__ void grad_kv(const GradDev& g, const Maps& there, const Maps& back, const GradPlace& where)
{
    using S = GradShape<DK, DV>;
    const AttnDev& p = g.f;
    const long long ci = where.chunk, at = ci * p.heads + where.head;
    const int head = where.head;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, quarter = warp % 4, sub = warp / 4;
    const Chunk c = chunk_at(p, ci);
    if (c.len <= 0)
        return;
    char* smem = dattn_tiles;
    typename S::Small& sm = *reinterpret_cast<typename S::Small*>(smem + S::TILES);
    const Decays& dec = sm.dec;
    char* s_keys = smem + S::K_BYTES;
    char* s_values = s_keys + S::K_BYTES;
    const uint32_t queries = __shfl_sync(0xffffffffu, smem_u32(smem), 0), keys = queries + S::K_BYTES, values = keys + S::K_BYTES, dys = values + S::V_BYTES,
                   image = dys + S::V_BYTES;
    const uint32_t tmem = begin_grad<T, DK, DV, true>(g, there, back, c, at, head, sm, queries);         // scores, v dy', dk, dv: 128 columns each
    const uint32_t scores = tmem, slopes = tmem + 128, dks = tmem + 256, dvs = tmem + 384, lanes = (uint32_t)(quarter * 32) << 16;
    if (warp == 0) {
        constexpr uint32_t id = instruction(kIsBf16<T>, false, false, 128, 128);
        if (elect_one()) {
            products<DV / 16, kColumns, kColumns>(slopes, over_columns(values, 0), over_columns(dys, 0), id, false);
            products<DK / 16, kColumns, kColumns>(scores, over_columns(keys, 0), over_columns(queries, 0), id, false);
            commit(smem_u32(&sm.ctl.bar[0]));
        }
        __syncwarp();
    }
    if (warp == 3) {                             // (of the last 32 tokens' warps, which have the fewest pairs to weigh, as warp 7)
        constexpr uint32_t id_k = instruction(kIsBf16<T>, false, false, 128, DK), id_v = instruction(kIsBf16<T>, false, true, 128, DV);
        await(smem_u32(&sm.image), 0, &sm.ctl.dead);
        __syncwarp();
        if (elect_one()) {
            products<DV / 16, kColumns, 2 * DK>(dks, over_columns(values, 0), image_over_dv<DK>(image + S::IMAGE, 0), id_k, false);
            commit(smem_u32(&sm.second_product));
            products<DV / 16, kColumns, 2 * DK>(dks, over_columns(values, 0), image_over_dv<DK>(image, 0), id_k, true);
            products<DK / 16, kColumns, 16>(dvs, over_columns(keys, 0), image_over_dk<DK>(image, 0), id_v, false);
            commit(smem_u32(&sm.ctl.bar[1]));
        }
        __syncwarp();
        if (g.terms == 3) {                      // the third term takes the second one's place
            await(smem_u32(&sm.second_product), 0, &sm.ctl.dead);
            __syncwarp();
            behind_barrier();
            if (elect_one()) {
                expect_bytes(smem_u32(&sm.third), S::IMAGE);
                fetch_bytes(image + S::IMAGE, g.image_Z + (at * 3 + 2) * S::IMAGE, S::IMAGE, smem_u32(&sm.third));
            }
            __syncwarp();
            await(smem_u32(&sm.third), 0, &sm.ctl.dead);
            __syncwarp();
            if (elect_one()) {
                products<DV / 16, kColumns, 2 * DK>(dks, over_columns(values, 0), image_over_dv<DK>(image + S::IMAGE, 0), id_k, true);
                commit(smem_u32(&sm.third_product));
            }
            __syncwarp();
        }
    } else if (warp == 7) {
        if (elect_one())
            fetch_next<DK, DV>(g, there, back);
        __syncwarp();
    }
    grad_products_done(sm.ctl, 0);
    const int row = quarter * 32 + lane;
    uint32_t packed_v[16], packed_k[16], diagonal_v[4], diagonal_k[4];
    float most_v = 0.f, most_k = 0.f, own_v = 0.f, own_k = 0.f, over_v = 0.f, over_k = 0.f, over_own_v = 0.f, over_own_k = 0.f;
    float col = 0.f;
    if (sub > quarter) {
        float v[32], w[32];
        tmem_ld32(scores + sub * 32 + lanes, v);
        tmem_ld32(slopes + sub * 32 + lanes, w);
        const float to_there = to_block(dec, row, sub) * p.scale;
#pragma unroll
        for (int j = 0; j < 32; j += 4) {        // M's column sums: the decay once, in front of the products' operands, which have it each
            const float4 h = *reinterpret_cast<const float4*>(sm.from + sub * 32 + j);
            col = fmaf(v[j] * w[j], h.x, col);
            col = fmaf(v[j + 1] * w[j + 1], h.y, col);
            col = fmaf(v[j + 2] * w[j + 2], h.z, col);
            col = fmaf(v[j + 3] * w[j + 3], h.w, col);
        }
        col *= to_there;
        decay_earlier(v, to_there, sm.from + sub * 32);
        decay_earlier(w, to_there, sm.from + sub * 32);
        pack_weights<T>(v, packed_v, most_v, over_v);
        pack_weights<T>(w, packed_k, most_k, over_k);
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            packed_v[j] = packed_k[j] = 0;
    }
    {
        const int first = sub * 8, from = quarter * 32 + first;
        const float own = dec.g[row], own_low = dec.low[row];
        float v[8], w[8];
        tmem_ld8(scores + from + lanes, v);
        tmem_ld8(slopes + from + lanes, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool later = first + j >= lane;
            const float d = ex2((dec.g[from + j] - own) + (dec.low[from + j] - own_low)) * p.scale;
            v[j] = later ? v[j] * d : 0.f;
            w[j] = later ? w[j] * d : 0.f;
        }
        pack_weights<T>(v, diagonal_v, own_v, over_own_v);
        pack_weights<T>(w, diagonal_k, own_k, over_own_k);
    }
    if (!kIsBf16<T>) {
        sm.most[0][sub][row] = fmaxf(most_v, own_v);
        sm.most[1][sub][row] = fmaxf(most_k, own_k);
    }
    before_barrier();
    asm volatile("bar.sync %0, 128;" :: "r"(1 + quarter) : "memory");
    behind_barrier();
    float up_v = 1.f, up_k = 1.f, down_v = 1.f, down_k = 1.f;
    if (!kIsBf16<T>) {
        const float unit = g.unit_Z[at];
        up_v = power_of_row(sm.most[0], row, unit, down_v);
        up_k = power_of_row(sm.most[1], row, unit, down_k);
        change_power(packed_v, up_v * over_v);
        change_power(packed_k, up_k * over_k);
        change_power(diagonal_v, up_v * over_own_v);
        change_power(diagonal_k, up_k * over_own_k);
        up_v *= unit, up_k *= unit;
    }
    if (sub != quarter) {
        tmem_st16(scores + sub * 16 + lanes, packed_v);
        tmem_st16(slopes + sub * 16 + lanes, packed_k);
    }
    tmem_st4(scores + quarter * 16 + sub * 4 + lanes, diagonal_v);
    tmem_st4(slopes + quarter * 16 + sub * 4 + lanes, diagonal_k);
    grad_products_done(sm.ctl, 1);
    if (g.terms == 3) {
        await(smem_u32(&sm.third_product), 0, &sm.ctl.dead);
        __syncwarp();
        behind_barrier();
    }
    const float f = to_end(dec, row);
    sm.dots[sub][row] = weigh_row<T, DK>(dks + lanes, s_keys, row, sub, f * up_k) * down_k;
    weigh_row<T, DV>(dvs + lanes, nullptr, row, sub, f * up_v);
    sm.sums[sub][row] = col;
    tmem_st_done();
    before_barrier();
    __syncthreads();
    if (warp == 0) {
        behind_barrier();
        constexpr uint32_t id_k = instruction(kIsBf16<T>, false, true, 128, DK), id_v = instruction(kIsBf16<T>, false, true, 128, DV);
        if (elect_one()) {
            products_tmem<8, kTokens>(dvs, scores, over_tokens(dys, 0), id_v);
            products_tmem<8, kTokens>(dks, slopes, over_tokens(queries, 0), id_k);
            commit(smem_u32(&sm.ctl.bar[2]));
        }
        __syncwarp();
    }
    if (sub == 0 && g.want_l) {
        const long long plane = (long long)p.heads * p.chunks * kChunk;
        float* to = g.tokens + ((long long)head * p.chunks + ci) * kChunk + row;
        to[2 * plane] = (sm.dots[0][row] + sm.dots[1][row]) + (sm.dots[2][row] + sm.dots[3][row]);
        to[3 * plane] = (sm.sums[0][row] + sm.sums[1][row]) + (sm.sums[2][row] + sm.sums[3][row]);
    }
    grad_products_done(sm.ctl, 2);
    // (results in float32 take the place of queries and keys; all tiles are done with)
    if (g.part_k)
        stage_part<DK>(dks + lanes, smem, row, sub, down_k);
    else if (g.dk.ptr)
        stage_row<T, DK>(dks + lanes, s_keys, row, sub, down_k);
    if (g.dv.ptr)
        stage_row<T, DV>(dvs + lanes, s_values, row, sub, down_v);
    end_grad(sm.ctl, tmem);
    if (g.part_k)
        store_part<DK>(smem, g.part_k + (packed_row(p, c, 0) * p.heads + head) * p.dk, (long long)p.heads * p.dk, c.len, p.dk);
    else if (g.dk.ptr)
        store_tile<T, DK, kGradThreads>(s_keys, g.dk, c, head, p.dk, g.vec_dk);
    if (g.dv.ptr)
        store_tile<T, DV, kGradThreads>(s_values, g.dv, c, head, p.dv, g.vec_dv);
}

// Both in one launch, side by side: the second one finds the tiles in L2.  4 x 1024 tokens of 16 heads of 128 x 128 take 76 us: a block has an SM's shared memory to itself and goes through
// loads (2200 clocks), products, weights, products and stores one behind the other, 12000 clocks for dq and 14000 for dk and dv.
template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kGradThreads, 1) grad_kernel(const __grid_constant__ Maps there, const __grid_constant__ Maps back, const GradDev g)
{
    wait_for_previous();
    const GradPlace where = grad_place(g, blockIdx.x);
    if (where.kv)
        grad_kv<T, DK, DV>(g, there, back, where);
    else
        grad_q<T, DK, DV>(g, there, back, where);
}

// exp(G_C) <Z, S_0> of each chunk and head from the images of both, where the walks ran side by side.
template <typename T>
__global__ void __launch_bounds__(kThreads) grad_across_kernel(const GradDev g, int image_bytes)
{
    wait_for_previous();
    __shared__ float s_sum[8];
    const AttnDev& p = g.f;
    const long long at = blockIdx.x;
    if (chunk_at(p, at / p.heads).len <= 0)
        return;
    const uint4* S = reinterpret_cast<const uint4*>(g.image_S + at * ((long long)g.terms * image_bytes));
    const uint4* Z = reinterpret_cast<const uint4*>(g.image_Z + at * ((long long)g.terms * image_bytes));
    float dot = 0.f;
#pragma unroll 2
    for (int i = threadIdx.x; i < image_bytes / 16; i += kThreads) {
        float a[8] = {}, b[8] = {};
#pragma unroll
        for (int t = 2; t >= 0; --t) {
            const uint4 x = load_if(S + t * (image_bytes / 16) + i, t < g.terms), y = load_if(Z + t * (image_bytes / 16) + i, t < g.terms);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 u = unpack16<T>((&x.x)[j]), v = unpack16<T>((&y.x)[j]);
                a[2 * j] += u.x, a[2 * j + 1] += u.y;
                b[2 * j] += v.x, b[2 * j + 1] += v.y;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            dot = fmaf(a[j], b[j], dot);
    }
#pragma unroll
    for (int o = 16; o; o /= 2)
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
    if (threadIdx.x % 32 == 0)
        s_sum[threadIdx.x / 32] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
        dot = 0.f;
        for (int i = 0; i < 8; ++i)
            dot += s_sum[i];
        g.across[at] = dot * g.whole[at] * (kIsBf16<T> ? 1.f : g.unit_S[at] * g.unit_Z[at]);
    }
}

// Sums of dq and dk over the heads of a group, in the order of the heads; V channels to a thread.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) grad_group_kernel(const GradDev g)
{
    wait_for_previous();
    const AttnDev& p = g.f;
    const Chunk c = chunk_at(p, blockIdx.x);
    const int each = p.dk / V, n = p.heads / p.share * each;
    const float* part = blockIdx.z ? g.part_k : g.part_q;
    if (!part)
        return;
    for (int e = blockIdx.y * kThreads + threadIdx.x; e < c.len * n; e += gridDim.y * kThreads) {
        const int t = e / n, i = e % n;
        const float* from = part + packed_row(p, c, t) * p.heads * p.dk + (long long)(i / each) * p.share * p.dk + i % each * V;
        float sum[V] = {};
#pragma unroll 4
        for (int h = 0; h < p.share; ++h) {
            const Vec<float, V> v = *reinterpret_cast<const Vec<float, V>*>(from + (long long)h * p.dk);
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[j] += v.v[j];
        }
        T* to = row_ptr<T>(blockIdx.z ? g.dk : g.dq, c.seq, c.row0 + t) + (long long)(i / each) * p.dk + i % each * V;
#pragma unroll
        for (int j = 0; j < V; ++j)
            to[j] = from_f<T>(sum[j]);
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
        float over = lane < g.across_of ? g.across[ch * g.across_of + lane] : 0.f;
#pragma unroll
        for (int o = 16; o; o /= 2)
            over += __shfl_xor_sync(0xffffffffu, over, o);
        over += block == 1 || block == 2 ? g.bridges[2 * ch + block - 1] : 0.f;
        const float A = rate(p, head);
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
            const bool none = dl[i] == 0.f;      // what is forgotten has no share, whatever forgets it (a step of infinity)
            const float d = none ? 0.f : dl[i] * A * slope;
            sum_A = none ? sum_A : fmaf(dl[i], step, sum_A);
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
