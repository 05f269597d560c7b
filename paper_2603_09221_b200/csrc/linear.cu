// Host side of ttc_linear and ttc_linear_grad.
#include <cuda.h>

#include <initializer_list>

#include "block_host.h"
#include "device_error.h"
#include "tensor_map.h"
#include "linear_rows.cuh"

using namespace ttc;
using namespace ttc::blk;
using namespace ttc::lin;

namespace {

// Rows up to which W is streamed past all of x (few_rows_kernel) instead of going through tiles of 128 rows.  2048 -> 4096,
// 1024 -> 1024 and 8192 -> 8192: 32 rows 9.3, 4.9 and 33.7 us, by tiles 11.2, 6.6 and 35.6; 64 rows 14.3, 8.2 and 58.6 (by a form for as
// many), by tiles 11.3, 6.7 and 35.5.  Rows that cannot be read by 16 bytes: 2047 -> 4095, 8 rows 15.8 us and 32 rows 39.5, against 34.5 for
// 64 rows by tiles, most of it the copies of W and x.
constexpr int kFewRows = 32;

// Parts of the contraction of few_rows_kernel, the blocks of a cluster: while all blocks are at work at once, two to an SM, and a part has 1024
// indices.  What a cluster costs is about 1.2 us: 8 rows, 4096 -> 2048 7.5 -> 6.4 us and 16 rows 16.9 -> 8.3 in 2 and 4 parts, but 1024 -> 1024
// 2.7 -> 3.9; twice as many blocks 8 rows, 2048 -> 4096 5.7 -> 9.3.
int few_parts(int64_t blocks, int64_t k, int sms)
{
    int parts = 1;
    while (parts < 8 && 2 * parts * blocks <= 2 * sms && k >= parts * 2 * 1024)
        parts *= 2;
    return parts;
}

// Matrix of `rows` rows of `cols` 16-bit elements, fetched in boxes of 64 columns (128 bytes, swizzled) by `box` rows.
int encode(CUtensorMap& map, const void* ptr, int64_t rows, int64_t cols, int64_t ld, int box, bool is_bf16)
{
    EncodeTiled f;
    TTC_TRY(encoder(f));
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, steps[2] = {1, 1};
    const CUresult r = f(&map, is_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(ptr), dims, strides,
                         boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? TTC_OK : fail(TTC_STATUS_CUDA_ERROR, "cuTensorMapEncodeTiled: error %d", (int)r);
}

bool aligned(const void* p, int64_t ld, size_t size) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (int64_t)size % 16 == 0; }

// Matrices of a call that share elements, or may (rows_overlap); of different types or numbers of rows: ranges that meet.
struct Matrix {
    const void* ptr;
    int64_t rows, cols, ld;
    size_t size;
    size_t bytes() const { return rows > 0 ? (size_t)((rows - 1) * ld + cols) * size : 0; }
};
bool meet(const Matrix& a, const Matrix& b)
{
    if (a.size != b.size || a.rows != b.rows)
        return ranges_meet(a.ptr, a.bytes(), b.ptr, b.bytes());
    return rows_overlap(ttc_rows{const_cast<void*>(a.ptr), 0, a.ld}, a.cols, ttc_rows{const_cast<void*>(b.ptr), 0, b.ld}, b.cols, 1, a.rows, false, a.size);
}

// An operand of a product in memory: `rows` rows of `cols` elements.
struct Operand {
    const void* ptr;
    int64_t rows, cols, ld;
};

// What TMA cannot read is copied into the workspace first.
struct Aligned {
    Operand from, to;
    bool copy;
};

Aligned plan_operand(const Operand& o, Scratch& s)
{
    Aligned r{o, o, false};
    if (!aligned(o.ptr, o.ld, 2)) {
        r.copy = true;
        r.to.ld = (o.cols + 7) / 8 * 8;
        r.to.ptr = s.take<unsigned short>((size_t)o.rows * r.to.ld);
    }
    return r;
}

int copy_operand(const Aligned& a, cudaStream_t st)
{
    if (!a.copy || a.from.rows == 0)
        return TTC_OK;
    return launch_early("projection, rows aligned", align_rows_kernel, dim3((unsigned)a.from.rows), 256, 0, 1, st,
                        static_cast<const unsigned short*>(a.from.ptr), a.from.ld, a.from.rows, (int)a.from.cols,
                        static_cast<unsigned short*>(const_cast<void*>(a.to.ptr)), a.to.ld);
}

// A product of `M` x `N` results over `K`: how it is tiled, and the scratch of a split contraction.
struct Product {
    int64_t M, N, K;
    int bn, splits;
    bool pair;                   // two CTAs on tiles of 256 x 256
    bool segments;               // added up in registers, every kSegment contraction indices
    float* part;
};

// Width of a tile and parts of the contraction.  A block of 64 contraction indices takes about 400 + 1.75 BN clocks: filling
// and reading its (128 + BN) x 128 bytes of shared memory, twice 128 + BN clocks, and what goes with it; so the width is the
// one with the least of that times the rounds of tiles over the SMs (512 x 4096 results over 2048 indices: 64 wide 19.7 us in two
// rounds, 128 wide in one 13.7).  In the same unit (a quarter of a clock) a pair's block costs kPairCost: 8192 x 2048 over 4096 97 us
// in pairs and 104 without, 4096 x 2048 over 2048 28.2 and 29.9, but 512 x 4096 over 2048 16.7 and 13.6, 1024 x 2304 over 1024 11.9 and 9.2.
constexpr int64_t kPairCost = 3050;
// Results with few tiles split the contraction too, in parts of at least 512 indices that a launch of its own sums.  That
// costs about 4 us, a block of 64 about 0.2: 64 x 2048 over 4096 (four parts) 18.6 -> 10.6 us, 256 x 2048 over 4096 (two) 19.0 -> 16.0, but
// 128 x 4096 over 2048 (two) 11.5 -> 12.5 and 64 x 1024 over 1024 6.7 -> 7.0; so as many blocks have to be saved:
constexpr int64_t kWorthSplit = 24;
// float32 results: contractions longer than kLong are added up in registers every kSegment indices.
constexpr int64_t kSegment = 512, kLong = 1024;

Product plan_product(int64_t M, int64_t N, int64_t K, bool f32, int sms, Scratch& s)
{
    Product p{M, N, K, 256, 1, false, f32 && K > kLong, nullptr};
    const int64_t tm = (M + BM - 1) / BM;
    int64_t least = INT64_MAX;
    for (int bn = p.segments ? 128 : 256; bn >= (p.segments ? 128 : 64); bn /= 2) {
        const int64_t rounds = (tm * ((N + bn - 1) / bn) + sms - 1) / sms, cost = rounds * (1600 + 7 * bn);
        if (cost < least) {
            least = cost;
            p.bn = bn;
        }
    }
    const int64_t pairs = sms / 2, rounds = ((M + 2 * BM - 1) / (2 * BM) * ((N + 255) / 256) + pairs - 1) / pairs;
    if (rounds * kPairCost < least) {
        p.pair = true;
        p.bn = 256;
        return p;
    }
    const int64_t tiles = tm * ((N + p.bn - 1) / p.bn), blocks = (K + BK - 1) / BK;
    int64_t splits = sms / tiles < K / 512 ? sms / tiles : K / 512;
    if (splits > 1 && blocks - blocks / splits >= kWorthSplit) {
        p.splits = (int)splits;
        p.part = s.take<float>((size_t)p.splits * M * N);
    }
    return p;
}

template <bool A_MN, bool B_MN, int BN, bool PAIR, bool SEGMENTS, typename OT>
int launch_tiles(const CUtensorMap& ma, const CUtensorMap& mb, GemmDev& g, bool is_bf16, int sms, cudaStream_t st)
{
    using S = GemmShape<BN, PAIR>;
    constexpr int CTAS = PAIR ? 2 : 1;
    auto* kernel = gemm_kernel<A_MN, B_MN, BN, PAIR, OT, SEGMENTS>;
    TTC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
    g.tiles_m = (int)((g.M + CTAS * BM - 1) / (CTAS * BM));
    g.tiles_n = (int)((g.N + BN - 1) / BN);
    g.idesc = instruction(is_bf16, A_MN, B_MN, CTAS * BM, BN);
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n * g.splits, most = sms / CTAS;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)(CTAS * (tiles < most ? tiles : most)));
    c.blockDim = dim3(kGemmThreads);
    c.dynamicSmemBytes = S::SMEM;
    c.stream = st;
    cudaLaunchAttribute with[2];
    with[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // (as launch_early)
    with[0].val.programmaticStreamSerializationAllowed = 1;
    with[1].id = cudaLaunchAttributeClusterDimension;
    with[1].val.clusterDim.x = CTAS;
    with[1].val.clusterDim.y = with[1].val.clusterDim.z = 1;
    c.attrs = with;
    c.numAttrs = PAIR ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, ma, mb, g);
    return e == cudaSuccess ? launched("matrix product") : fail(TTC_STATUS_CUDA_ERROR, "matrix product: %s", cudaGetErrorString(e));
}

// D = A B' with A [M][K] (or [K][M] with A_MN) and B likewise, and the epilogue on it.
template <bool A_MN, bool B_MN> int product(const Product& q, const Operand& a, const Operand& b, bool is_bf16, int out_dtype, const Epilogue& e, int sms, cudaStream_t st)
{
    CUtensorMap ma, mb;
    TTC_TRY(encode(ma, a.ptr, a.rows, a.cols, a.ld, A_MN ? BK : BM, is_bf16));
    TTC_TRY(encode(mb, b.ptr, b.rows, b.cols, b.ld, B_MN ? BK : q.pair ? q.bn / 2 : q.bn, is_bf16));
    GemmDev g = {};
    g.M = q.M;
    g.N = q.N;
    g.k_blocks = (int)((q.K + BK - 1) / BK);
    g.splits = q.splits;
    g.segment = kSegment / BK;
    g.e = e;
    if (q.splits > 1) {
        g.e = Epilogue{};
        g.e.out = q.part;
        g.e.ldo = q.N;
        g.e.split_stride = q.M * q.N;
        g.e.vec_o = q.N % 4 == 0;
    }
    const int type = q.splits > 1 ? (int)TTC_F32 : out_dtype;
    TTC_TRY(by_type(type, [&](auto t) {
        using OT = decltype(t);
        if constexpr (!A_MN && !B_MN && sizeof(OT) == 4)             // (only the forward product has float32 results)
            if (q.segments)
                return q.pair ? launch_tiles<A_MN, B_MN, 256, true, true, OT>(ma, mb, g, is_bf16, sms, st)
                              : launch_tiles<A_MN, B_MN, 128, false, true, OT>(ma, mb, g, is_bf16, sms, st);
        if (q.pair)
            return launch_tiles<A_MN, B_MN, 256, true, false, OT>(ma, mb, g, is_bf16, sms, st);
        switch (q.bn) {
        case 256: return launch_tiles<A_MN, B_MN, 256, false, false, OT>(ma, mb, g, is_bf16, sms, st);
        case 128: return launch_tiles<A_MN, B_MN, 128, false, false, OT>(ma, mb, g, is_bf16, sms, st);
        default: return launch_tiles<A_MN, B_MN, 64, false, false, OT>(ma, mb, g, is_bf16, sms, st);
        }
    }));
    if (q.splits == 1)
        return TTC_OK;
    return by_type(out_dtype, [&](auto t) {
        using OT = decltype(t);
        const unsigned blocks = (unsigned)((q.M * q.N + 255) / 256);
        auto* kernel = is_bf16 ? split_sum_kernel<bf16, OT> : split_sum_kernel<__half, OT>;
        return launch_early("matrix product, parts of the contraction", kernel, dim3(blocks), 256, 0, 1, st, q.part, q.M * q.N, q.splits, q.M, q.N, e);
    });
}

int check(const ttc_linear_args* a)
{
    if (!a)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "arguments are null");
    TTC_TRY(check_dtype(a->dtype, false));
    if (a->out_dtype != a->dtype && a->out_dtype != TTC_F32)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "output type %d for operands of type %d", a->out_dtype, a->dtype);
    if (a->rows < 0 || a->k < 1 || a->m < 1)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "rows = %lld, k = %d, m = %d", (long long)a->rows, a->k, a->m);
    if (a->rows > kMaxRows || a->k > kMaxRows || a->m > kMaxRows)
        return fail(TTC_STATUS_UNSUPPORTED, "rows = %lld, k = %d, m = %d", (long long)a->rows, a->k, a->m);
    if (a->act < TTC_ACT_NONE || a->act > TTC_ACT_SOFTPLUS)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "activation %d", a->act);
    TTC_TRY(check_floats("x", a->x, a->rows == 0, 2));
    TTC_TRY(check_floats("w", a->w, false, 2));
    TTC_TRY(check_floats("bias", a->bias, true));
    TTC_TRY(check_floats("pre", a->pre, true, 2));
    if ((a->rows > 1 && a->ldx < a->k) || a->ldw < (a->m > 1 ? a->k : 0) || (a->pre && a->rows > 1 && a->ldp < a->m))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "row strides shorter than the rows");
    return TTC_OK;
}

struct LinearPlan {
    bool few;
    Aligned x, w;
    Product q;
    size_t bytes;
};

int plan_linear(int device, const ttc_linear_args* a, void* ws, LinearPlan& o)
{
    TTC_TRY(check(a));
    const size_t size = element_size(a->out_dtype);
    TTC_TRY(check_floats("y", a->y, a->rows == 0, size));
    TTC_TRY(check_floats("residual", a->residual, true, size));
    if (a->rows > 1 && (a->ldy < a->m || (a->residual && a->ldr < a->m)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "row strides shorter than the rows");
    const Matrix y{a->y, a->rows, a->m, a->ldy, size}, pre{a->pre, a->rows, a->m, a->ldp, 2}, r{a->residual, a->rows, a->m, a->ldr, size};
    for (const Matrix& in : {Matrix{a->x, a->rows, a->k, a->ldx, 2}, Matrix{a->w, a->m, a->k, a->ldw, 2}})
        if (meet(y, in) || meet(pre, in))
            return fail(TTC_STATUS_INVALID_ARGUMENT, "y or pre overlaps x or w");
    const bool in_place = a->y == a->residual && (a->rows == 1 || a->ldy == a->ldr);
    if (meet(pre, y) || meet(pre, r) || (!in_place && meet(y, r)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "y, pre and parts of residual overlap");
    const int64_t ldx = a->rows > 1 ? a->ldx : (a->k + 7) / 8 * 8, ldw = a->m > 1 ? a->ldw : (a->k + 7) / 8 * 8;
    Scratch s(ws);
    o.few = a->rows <= kFewRows;
    o.x = Aligned{Operand{a->x, a->rows, a->k, ldx}, Operand{a->x, a->rows, a->k, ldx}, false};
    o.w = Aligned{Operand{a->w, a->m, a->k, ldw}, Operand{a->w, a->m, a->k, ldw}, false};
    if (!o.few) {
        o.x = plan_operand(o.x.from, s);
        o.w = plan_operand(o.w.from, s);
        o.q = plan_product(a->rows, a->m, a->k, a->out_dtype == TTC_F32, sm_count(device), s);
    }
    o.bytes = s.used;
    return TTC_OK;
}

struct GradPlan {
    Aligned x, w, dz;            // dz: dy itself where it can be used as it is
    SlopeDev slope;
    int slope_v, row_blocks;
    bool need_slope;
    Product qx, qw;
    size_t bytes;
};

int plan_grad(int device, const ttc_linear_args* a, const ttc_linear_grads* g, void* ws, GradPlan& o)
{
    TTC_TRY(check(a));
    if (!g)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "gradients are null");
    const size_t size = element_size(a->out_dtype);
    TTC_TRY(check_floats("dy", g->dy, a->rows == 0, size));
    TTC_TRY(check_floats("dx", g->dx, true, 2));
    TTC_TRY(check_floats("dw", g->dw, true, 2));
    TTC_TRY(check_floats("dbias", g->dbias, true));
    if (a->act != TTC_ACT_NONE && !a->pre && a->rows)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "pre is null: the gradients of an activation need it");
    if ((a->rows > 1 && (g->lddy < a->m || (g->dx && g->lddx < a->k))) || (g->dw && a->m > 1 && g->lddw < a->k))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "row strides shorter than the rows");
    const Matrix dx{g->dx, a->rows, a->k, g->lddx, 2}, dw{g->dw, a->m, a->k, g->lddw, 2};
    for (const Matrix& in : {Matrix{a->x, a->rows, a->k, a->ldx, 2}, Matrix{a->w, a->m, a->k, a->ldw, 2}, Matrix{g->dy, a->rows, a->m, g->lddy, size},
                             Matrix{a->act == TTC_ACT_NONE ? nullptr : a->pre, a->rows, a->m, a->ldp, 2}})
        if (meet(dx, in) || meet(dw, in))
            return fail(TTC_STATUS_INVALID_ARGUMENT, "dx or dw overlaps an input");
    if (meet(dx, dw))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dx and dw overlap");
    const int sms = sm_count(device);
    const int64_t ldx = a->rows > 1 ? a->ldx : (a->k + 7) / 8 * 8, ldw = a->m > 1 ? a->ldw : (a->k + 7) / 8 * 8;
    const int64_t lddy = a->rows > 1 ? g->lddy : (a->m + 7) / 8 * 8;
    Scratch s(ws);
    o = GradPlan{};
    SlopeDev& d = o.slope;
    d.rows = a->rows;
    d.m = a->m;
    d.dy = g->dy;
    d.pre = a->pre;
    d.lddy = lddy;
    d.ldp = a->rows > 1 ? a->ldp : 0;
    const bool products = g->dx || g->dw;
    o.dz.from = o.dz.to = Operand{g->dy, a->rows, a->m, lddy};
    const bool as_it_is = a->act == TTC_ACT_NONE && a->out_dtype == a->dtype && aligned(g->dy, lddy, 2);
    if (products && !as_it_is) {
        d.lddz = (a->m + 7) / 8 * 8;
        d.dz = s.take<unsigned short>((size_t)a->rows * d.lddz);
        o.dz.to = Operand{d.dz, a->rows, a->m, d.lddz};
    }
    o.need_slope = (products && !as_it_is) || g->dbias;
    // eight columns to a thread where everything allows 16-byte accesses
    const bool wide = a->m % 8 == 0 && aligned(g->dy, lddy, size) && (a->act == TTC_ACT_NONE || aligned(a->pre, d.ldp, 2));
    o.slope_v = wide ? 8 : 1;
    const int64_t cols = (a->m + 32 * o.slope_v - 1) / (32 * o.slope_v);
    int64_t per = 256;
    while (per > 16 && cols * ((a->rows + per - 1) / per) < 4 * (int64_t)sms)
        per /= 2;
    while ((a->rows + per - 1) / per > kMaxGridY)
        per *= 2;
    d.rows_per_block = (int)per;
    o.row_blocks = (int)((a->rows + per - 1) / per);
    if (g->dbias)
        d.part = s.take<float>((size_t)o.row_blocks * a->m);
    if (g->dw)
        o.x = plan_operand(Operand{a->x, a->rows, a->k, ldx}, s);
    if (g->dx)
        o.w = plan_operand(Operand{a->w, a->m, a->k, ldw}, s);
    // the two products run one behind the other and share the room for parts
    Scratch s1 = s, s2 = s;
    if (g->dx && a->rows)                        // (no rows: no products, and no tiles to share the SMs out to)
        o.qx = plan_product(a->rows, a->k, a->m, false, sms, s1);
    if (g->dw && a->rows)
        o.qw = plan_product(a->m, a->k, a->rows, false, sms, s2);
    o.bytes = s1.used > s2.used ? s1.used : s2.used;
    return TTC_OK;
}

} // namespace

extern "C" {

int64_t ttc_linear_workspace(int32_t device, const ttc_linear_args* a)
{
    LinearPlan o;
    TTC_TRY(plan_linear(device, a, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_linear(int32_t device, const ttc_linear_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    LinearPlan o;
    TTC_TRY(plan_linear(device, a, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (a->rows == 0)
        return TTC_OK;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool is_bf16 = a->dtype == TTC_BF16;
    const size_t size = element_size(a->out_dtype);
    Epilogue e = {};
    e.out = a->y;
    e.ldo = a->ldy;
    e.bias = a->bias;
    e.residual = a->residual;
    e.ldr = a->ldr;
    e.pre = a->pre;
    e.ldp = a->ldp;
    e.act = a->act;
    e.pre_bf16 = is_bf16;
    e.vec_o = aligned(a->y, a->ldy, size);
    e.vec_r = aligned(a->residual, a->ldr, size);
    e.vec_p = aligned(a->pre, a->ldp, 2);
    if (o.few) {
        FewDev f = {};
        f.x = a->x;
        f.w = a->w;
        f.ldx = o.x.from.ld;
        f.ldw = o.w.from.ld;
        f.rows = (int)a->rows;
        f.k = a->k;
        f.m = a->m;
        f.vec = a->k % 8 == 0 && aligned(a->x, f.ldx, 2) && aligned(a->w, f.ldw, 2);
        f.e = e;
        return by_type(a->out_dtype, [&](auto t) {
            using OT = decltype(t);
            auto go = [&](auto tc, auto nt) {
                using T = decltype(tc);
                constexpr int NT = decltype(nt)::value, COLS = FewShape<NT>::COLS;
                const int blocks = (a->m + COLS - 1) / COLS;
                const int parts = few_parts(blocks, a->k, sm_count(device));
                f.part = (a->k + 256 * parts - 1) / (256 * parts) * 256;
                static std::atomic<uint64_t> allowed;                // devices, a bit each, that know of its shared memory
                const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
                if (FewShape<NT>::RING && !(allowed.load(std::memory_order_relaxed) & bit)) {
                    TTC_CUDA(cudaFuncSetAttribute(few_rows_kernel<T, OT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewShape<NT>::SMEM));
                    allowed.fetch_or(bit, std::memory_order_relaxed);
                }
                return launch_early("projection of few rows", few_rows_kernel<T, OT, NT>, dim3(blocks, parts), kFewWarps * 32, FewShape<NT>::SMEM, parts, st, f);
            };
            auto by_rows = [&](auto tc) {
                return a->rows <= 8 ? go(tc, std::integral_constant<int, 1>()) : a->rows <= 16 ? go(tc, std::integral_constant<int, 2>())
                                                                                             : go(tc, std::integral_constant<int, 4>());
            };
            return is_bf16 ? by_rows(bf16()) : by_rows(__half());
        });
    }
    TTC_TRY(copy_operand(o.x, st));
    TTC_TRY(copy_operand(o.w, st));
    return product<false, false>(o.q, o.x.to, o.w.to, is_bf16, a->out_dtype, e, sm_count(device), st);
}

int64_t ttc_linear_grad_workspace(int32_t device, const ttc_linear_args* a, const ttc_linear_grads* g)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_linear_grad(int32_t device, const ttc_linear_args* a, const ttc_linear_grads* g, void* workspace,
                    int64_t workspace_bytes, void* cuda_stream)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool is_bf16 = a->dtype == TTC_BF16;
    const int sms = sm_count(device);
    if (a->rows == 0) {                                              // sums over no rows
        if (g->dbias)
            TTC_CUDA(cudaMemsetAsync(g->dbias, 0, sizeof(float) * a->m, st));
        if (g->dw) {
            TTC_TRY((launch_early("gradients of a projection without rows", zero_rows_kernel<bf16>, dim3((unsigned)a->m), 256, 0, 1, st, static_cast<bf16*>(g->dw),
                                  g->lddw, a->m, a->k)));            // zero has the same bits in both types
        }
        return TTC_OK;
    }
    if (o.need_slope) {
        TTC_TRY(by_type(a->out_dtype, [&](auto t) {
            using OT = decltype(t);
            const dim3 grid((unsigned)((a->m + 32 * o.slope_v - 1) / (32 * o.slope_v)), (unsigned)o.row_blocks);
            auto go = [&](auto tc) {
                using T = decltype(tc);
                auto with = [&](auto act) {
                    constexpr int ACT = decltype(act)::value;
                    auto* kernel = o.slope_v == 8 ? slope_kernel<T, OT, 8, ACT> : slope_kernel<T, OT, 1, ACT>;
                    kernel<<<grid, 256, 0, st>>>(o.slope);
                    return launched("gradients of a projection, activation");
                };
                switch (a->act) {
                case TTC_ACT_RELU: return with(std::integral_constant<int, TTC_ACT_RELU>());
                case TTC_ACT_SILU: return with(std::integral_constant<int, TTC_ACT_SILU>());
                case TTC_ACT_GELU: return with(std::integral_constant<int, TTC_ACT_GELU>());
                case TTC_ACT_SOFTPLUS: return with(std::integral_constant<int, TTC_ACT_SOFTPLUS>());
                default: return with(std::integral_constant<int, TTC_ACT_NONE>());
                }
            };
            return is_bf16 ? go(bf16()) : go(__half());
        }));
        if (g->dbias) {
            TTC_TRY((launch_early("gradients of a projection, bias", bias_sum_kernel, dim3((a->m + 31) / 32), 256, 0, 1, st, o.slope.part, o.row_blocks, a->m, g->dbias)));
        }
    }
    if (g->dx) {
        TTC_TRY(copy_operand(o.w, st));
        Epilogue e = {};
        e.out = g->dx;
        e.ldo = a->rows > 1 ? g->lddx : 0;
        e.vec_o = aligned(g->dx, e.ldo, 2);
        TTC_TRY((product<false, true>(o.qx, o.dz.to, o.w.to, is_bf16, a->dtype, e, sms, st)));
    }
    if (g->dw) {
        TTC_TRY(copy_operand(o.x, st));
        Epilogue e = {};
        e.out = g->dw;
        e.ldo = g->lddw;
        e.vec_o = aligned(g->dw, e.ldo, 2);
        TTC_TRY((product<true, true>(o.qw, o.dz.to, o.x.to, is_bf16, a->dtype, e, sms, st)));
    }
    return TTC_OK;
}

int ttc_block_device_error(int32_t device, int32_t* value)
{
    if (!value)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "value is null");
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    int v = 0;
    int w = 0;
    TTC_CUDA(cudaMemcpyFromSymbol(&v, g_error, sizeof(v)));
    TTC_TRY(attention_device_error(&w));
    *value = v | w;
    return TTC_OK;
}

} // extern "C"
