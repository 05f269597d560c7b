// Host side of ttc_decay_attention, ttc_decay_attention_step and ttc_decay_attention_grad.
#include <algorithm>
#include <type_traits>

#include "block_host.h"
#include "decay_attention_grad.cuh"
#include "device_error.h"
#include "tensor_map.h"

using namespace ttc;
using namespace ttc::blk;
using namespace ttc::dattn;

namespace {

int check(const ttc_decay_args* a, bool step)
{
    if (!a)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "arguments are null");
    TTC_TRY(check_dtype(a->dtype, false));
    TTC_TRY(check_sequences(a->batch, step ? 1 : a->tokens, step ? nullptr : a->seq_offsets));
    if (a->heads < 1 || a->groups < 1 || a->heads % a->groups || a->dk < 1 || a->dv < 1)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "heads = %d, groups = %d, dk = %d, dv = %d", a->heads, a->groups, a->dk, a->dv);
    if (a->dk > 128 || a->dv > 128)
        return fail(TTC_STATUS_UNSUPPORTED, "dk = %d, dv = %d: 1 to 128 channels of a head are served", a->dk, a->dv);
    if (a->heads > kMaxGridY || a->batch > INT32_MAX / a->heads)
        return fail(TTC_STATUS_UNSUPPORTED, "batch = %lld, heads = %d", (long long)a->batch, a->heads);
    if (!(a->scale > -3.4e38f && a->scale < 3.4e38f))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "scale is not finite");
    const bool none = a->batch == 0 || (!step && a->tokens == 0);    // no rows, no addresses
    TTC_TRY(check_rows("q", a->q, a->dtype, none));
    TTC_TRY(check_rows("k", a->k, a->dtype, none));
    TTC_TRY(check_rows("v", a->v, a->dtype, none));
    TTC_TRY(check_rows("delta", a->delta, a->dtype, true));
    TTC_TRY(check_floats("A", a->A, false));
    TTC_TRY(check_floats("delta_bias", a->delta_bias, true));
    TTC_TRY(check_floats("state", a->state, true));
    return check_floats("state_out", a->state_out, true);
}

bool same_rows(const ttc_rows& a, const ttc_rows& b) { return a.ptr == b.ptr && a.tstride == b.tstride && a.bstride == b.bstride; }

size_t state_bytes(const ttc_decay_args* a) { return (size_t)a->batch * a->heads * a->dk * a->dv * sizeof(float); }

int check_output(const ttc_decay_args* a, bool step)
{
    if (!step && a->state != a->state_out && ranges_meet(a->state, state_bytes(a), a->state_out, state_bytes(a)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "state_out overlaps parts of state");
    TTC_TRY(check_rows("y", a->y, a->dtype, a->batch == 0 || (!step && a->tokens == 0)));
    const int64_t tokens = step ? 1 : a->tokens, shared = (int64_t)a->groups * a->dk, values = (int64_t)a->heads * a->dv;
    const bool packed = !step && a->seq_offsets;
    auto clash = [&](const ttc_rows& r, int64_t width) { return rows_overlap(a->y, values, r, width, a->batch, tokens, packed, element_size(a->dtype)); };
    if ((clash(a->v, values) && !same_rows(a->y, a->v)) || clash(a->q, shared) || clash(a->k, shared) || clash(a->delta, a->heads))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "y overlaps q, k, delta or parts of v");
    return TTC_OK;
}

// Bytes that rows of heads of `width` elements can be accessed by.  (4 x 1024 tokens, 16 heads of 36 x 36, results written by 8 and by 2: 48 and 60 us; gradients 121 and 141.)
int bytes_at_once(const Rows& r, int width)
{
    for (int n : {8, 4})
        if (width % n == 0 && reinterpret_cast<uintptr_t>(r.ptr) % (2 * n) == 0 && r.ts % n == 0 && r.bs % n == 0)
            return 2 * n;
    return 2;
}
bool floats_by_16_bytes(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int padded(int d) { return d > 64 ? 128 : 64; }

template <typename F> int by_widths(const ttc_decay_args* a, F&& f)
{
    constexpr std::integral_constant<int, 64> small;
    constexpr std::integral_constant<int, 128> large;
    auto of_16_bits = [&](auto t) {
        if (a->dk > 64)
            return a->dv > 64 ? f(t, large, large) : f(t, large, small);
        return a->dv > 64 ? f(t, small, large) : f(t, small, small);
    };
    return a->dtype == TTC_BF16 ? of_16_bits(bf16()) : of_16_bits(__half());
}

AttnDev to_dev(const ttc_decay_args* a, bool step)
{
    AttnDev p = {};
    const int32_t* off = step ? nullptr : a->seq_offsets;
    p.seqs = Seqs{off, a->batch, step ? 1 : a->tokens};
    p.heads = a->heads;
    p.share = a->heads / a->groups;
    p.dk = a->dk;
    p.dv = a->dv;
    p.softplus = a->softplus;
    p.scale = a->scale;
    p.q = dev_rows(a->q, off);
    p.k = dev_rows(a->k, off);
    p.v = dev_rows(a->v, off);
    p.delta = dev_rows(a->delta, off);
    p.y = dev_rows(a->y, off);
    p.head_q = p.head_k = a->dk;
    p.head_v = a->dv;
    p.vec_y = bytes_at_once(p.y, a->dv);
    p.vec_state = a->dv % 8 == 0 && floats_by_16_bytes(a->state) && floats_by_16_bytes(a->state_out);
    p.A = a->A;
    p.delta_bias = a->delta_bias;
    p.state = a->state;
    p.state_out = a->state_out;
    p.chunks_per_seq = (p.seqs.tokens + kChunk - 1) / kChunk;
    p.chunks = off ? p.seqs.tokens / kChunk + a->batch : a->batch * p.chunks_per_seq;
    return p;
}

struct Plan {
    AttnDev p;
    Operands o;
    States q;
    int splits;
    size_t bytes;
};

int map_pieces(const AttnDev& p, int64_t piece, int at_least, int64_t bound, cudaStream_t st)
{
    if (!p.piece_map)
        return TTC_OK;
    return launch_early("decay attention, pieces", piece_map_kernel, dim3(1), 1024, 0, 1, st, p.seqs, (long long)piece, at_least, (long long)bound,
                        const_cast<int2*>(p.piece_map), const_cast<int*>(p.seq_first));
}

// Rows of heads as [batch][tokens][heads][width], in boxes of 64 channels (128 bytes, swizzled) of 128 tokens.
int describe(CUtensorMap& map, const Rows& r, int heads, int width, int head, const Seqs& s, bool is_bf16)
{
    if (!s.tokens || !s.batch)                   // nothing is read
        return TTC_OK;
    EncodeTiled f;
    TTC_TRY(encoder(f));
    const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)heads, (cuuint64_t)s.tokens, (cuuint64_t)(s.offsets ? 1 : s.batch)};
    // (the copy engine takes no stride of nothing, which is what a dimension of one may have)
    const cuuint64_t next = (cuuint64_t)head * 2, token = r.ts ? r.ts * 2 : next, seq = !s.offsets && r.bs ? r.bs * 2 : token;
    const cuuint64_t strides[3] = {next, token, seq};
    const cuuint32_t box[4] = {64, 1, kChunk, 1}, steps[4] = {1, 1, 1, 1};
    const CUresult e = f(&map, is_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, r.ptr, dims, strides, box, steps,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return e == CUDA_SUCCESS ? TTC_OK : fail(TTC_STATUS_CUDA_ERROR, "cuTensorMapEncodeTiled: error %d", (int)e);
}

// Rows that no map describes are laid out anew in scratch.
void align(const Seqs& s, int heads, int width, Rows& r, int& head, Operands& o, Scratch& scratch)
{
    const long long most = 1ll << 38;            // of strides in elements
    const int vec = bytes_at_once(r, width);             // (rows that lie over one another are not asked of the copy engine either)
    if (!s.tokens || !s.batch || (vec == 16 && (r.ts >= (long long)heads * width || s.tokens <= 1) && (s.offsets || r.bs || s.batch <= 1) && r.ts < most && r.bs < most))
        return;
    const int padded = (width + 7) / 8 * 8;
    const long long row = (long long)heads * padded;
    unsigned short* to = scratch.take<unsigned short>((size_t)(s.offsets ? s.tokens : s.batch * s.tokens) * row);
    auto& q = o.of[o.n++];
    q.from = r;
    q.to = to;
    q.heads = heads, q.width = width, q.padded = head = padded;
    q.vec = vec == 2 ? 2 : 8;
    r = Rows{to, s.offsets ? 0 : s.tokens * row, row};
}
int align_all(const Seqs& s, const Operands& o, cudaStream_t st)
{
    if (!o.n)
        return TTC_OK;
    const long long rows = s.offsets ? s.tokens : s.batch * s.tokens;
    return launch_early("decay attention, rows laid out anew", align_kernel, dim3((unsigned)std::min((rows + kAlignRows - 1) / kAlignRows, (long long)kMaxGridY), o.n), 256, 0, 1, st, s, o);
}

// One walk to each sequence, head and `columns` value channels, or, where those leave SMs idle, to each of a sequence's pieces, behind a walk for what the pieces add to the state.  Uncut,
// n chunks take 2.65 n + 7 us; cut, the longest piece's m take 4.6 m + 25, so that n has to be above 7 m / 4 + 6.5.  (One sequence of 32 chunks, 128 x 128, uncut and cut: 64 walks, m = 16, 90 and 99 us;
// 48 walks, m = 11, 90 and 79; of 64 x 64, 36 walks, m = 8, 86 and 63; three of 8 chunks, 48 walks, m = 3, 29 and 38.)  Lengths of packed sequences are not known here: the longest is taken for
// one and a half times the mean (four in 32 chunks, 64 walks, m = 4: the longest of 15 chunks 49 and 48 us, of 9 chunks 35 and 50).
int take_pieces(int device, const ttc_decay_args* a, int splits, int columns, AttnDev& p, States& q, int ways, Scratch& s)
{
    const int64_t sms = sm_count(device), walks = (int64_t)a->heads * splits, rows = a->seq_offsets ? a->tokens : a->tokens * a->batch;
    const int64_t want = sms / walks;                                // pieces in all
    p.piece = a->tokens ? a->tokens : 1;
    p.pieces_per_seq = 1;
    p.pieces = a->batch;
    if (want > a->batch && a->batch && rows) {
        const int64_t each = want / a->batch;                        // of equal sequences, as many to each
        int64_t piece = a->seq_offsets ? (rows + want - 1) / want : (a->tokens + each - 1) / each;
        piece = (piece + kChunk - 1) / kChunk * kChunk;
        const int64_t longest = a->seq_offsets ? std::min(a->tokens, 3 * rows / (2 * a->batch)) : a->tokens;
        if (piece < a->tokens && 4 * longest > 7 * piece + 26 * kChunk) {
            p.piece = piece;
            p.pieces_per_seq = (a->tokens + piece - 1) / piece;
            p.pieces = a->seq_offsets ? a->tokens / piece + a->batch : a->batch * p.pieces_per_seq;
        }
    }
    if (p.pieces > INT32_MAX / (2 * walks))      // blocks are counted in 32 bits
        return fail(TTC_STATUS_UNSUPPORTED, "%lld pieces of sequences, %d heads", (long long)p.pieces, a->heads);
    if (p.piece < a->tokens) {
        for (int i = 0; i < ways; ++i) {
            q.way[i].piece_state = s.take<float>((size_t)p.pieces * a->heads * splits * kWalkThreads * (columns / 4));
            q.way[i].piece_decay = s.take<float>((size_t)p.pieces * a->heads);
        }
        p.piece_state = q.way[0].piece_state;
    }
    return TTC_OK;
}

int plan_forward(int device, const ttc_decay_args* a, void* ws, Plan& o)
{
    TTC_TRY(check(a, false));
    AttnDev& p = o.p;
    p = to_dev(a, false);
    o.splits = (a->dv + kCols - 1) / kCols;
    Scratch s(ws);
    o.o.n = 0;
    align(p.seqs, a->groups, a->dk, p.q, p.head_q, o.o, s);
    align(p.seqs, a->groups, a->dk, p.k, p.head_k, o.o, s);
    align(p.seqs, a->heads, a->dv, p.v, p.head_v, o.o, s);
    o.q = States{};
    TTC_TRY(take_pieces(device, a, o.splits, kCols, p, o.q, 1, s));
    o.bytes = s.used;
    return TTC_OK;
}

template <typename K> int allow_smem(K* kernel, int bytes)
{
    TTC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return TTC_OK;
}

// What the pieces add to the state, and from that the states in front of them (back: behind); `ways` walks in one launch.
template <typename T, int DK, int COLS> int piece_states(const Maps (&maps)[2], const AttnDev& p, States q, int ways, int splits, cudaStream_t st)
{
    q.way[0].image = q.way[1].image = nullptr;
    q.way[0].other = q.way[1].other = nullptr;   // (which nobody has written yet)
    q.ways = ways;
    const dim3 grid((unsigned)(p.pieces * p.heads * splits * ways));
    constexpr int smem = StateShape<T, DK, COLS>::SMEM;
    TTC_TRY((allow_smem(state_walk_kernel<T, DK, COLS>, smem)));
    TTC_TRY((launch_early("decay attention, what the pieces add", state_walk_kernel<T, DK, COLS>, grid, kWalkBlock, smem, 1, st, maps[0], maps[1], p, q, splits)));
    return launch_early("decay attention, states of the pieces", join_kernel, dim3((unsigned)p.pieces, (unsigned)p.heads, (unsigned)(splits * ways * (COLS / 16))), kWalkThreads, 0, 1, st, p, q, COLS / 4, splits);
}

// The states in front of all chunks, and the gradients of those behind them, side by side or one after the other.
template <typename T, int DK, int COLS> int chunk_states(const Maps (&maps)[2], const AttnDev& p, const States& q, int splits, bool together, cudaStream_t st)
{
    if (p.pieces == 0)
        return TTC_OK;
    if (q.way[0].piece_state)
        TTC_TRY((piece_states<T, DK, COLS>(maps, p, q, 2, splits, st)));
    constexpr int smem = StateShape<T, DK, COLS>::SMEM;
    TTC_TRY((allow_smem(state_walk_kernel<T, DK, COLS>, smem)));
    const unsigned walks = (unsigned)(p.pieces * p.heads * splits);
    States there = q;
    if (together) {
        there.ways = 2;
        return launch_early("decay attention, states and their gradients", state_walk_kernel<T, DK, COLS>, dim3(2 * walks), kWalkBlock, smem, 1, st, maps[0], maps[1], p, there, splits);
    }
    there.ways = 1;
    TTC_TRY((launch_early("decay attention, states", state_walk_kernel<T, DK, COLS>, dim3(walks), kWalkBlock, smem, 1, st, maps[0], maps[0], p, there, splits)));
    States back = there;
    back.way[0] = q.way[1];
    return launch_early("decay attention, gradients of states", state_walk_kernel<T, DK, COLS>, dim3(walks), kWalkBlock, smem, 1, st, maps[1], maps[1], p, back, splits);
}

struct GradPlan {
    GradDev g;
    Operands o;
    States q;
    int splits;
    bool together;
    size_t bytes;
};

int plan_grad(int device, const ttc_decay_args* a, const ttc_decay_grads* g, void* ws, GradPlan& o)
{
    TTC_TRY(check(a, false));
    if (!g)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "gradients are null");
    const int64_t shared = (int64_t)a->groups * a->dk, values = (int64_t)a->heads * a->dv;
    const struct { const char* name; const ttc_rows* r; int64_t width; } outs[] = {
        {"dq", &g->dq, shared}, {"dk", &g->dk, shared}, {"dv", &g->dv, values}, {"ddelta", &g->ddelta, a->heads}};
    const struct { const ttc_rows* r; int64_t width; } ins[] = {
        {&g->dy, values}, {&a->q, shared}, {&a->k, shared}, {&a->v, values}, {&a->delta, a->heads}};
    TTC_TRY(check_rows("dy", g->dy, a->dtype, a->batch == 0 || a->tokens == 0));
    const size_t size = element_size(a->dtype);
    for (int i = 0; i < 4; ++i) {
        TTC_TRY(check_rows(outs[i].name, *outs[i].r, a->dtype, true));
        for (auto& in : ins)
            if (rows_overlap(*outs[i].r, outs[i].width, *in.r, in.width, a->batch, a->tokens, a->seq_offsets, size))
                return fail(TTC_STATUS_INVALID_ARGUMENT, "%s overlaps an input", outs[i].name);
        for (int j = 0; j < i; ++j)
            if (rows_overlap(*outs[i].r, outs[i].width, *outs[j].r, outs[j].width, a->batch, a->tokens, a->seq_offsets, size))
                return fail(TTC_STATUS_INVALID_ARGUMENT, "%s overlaps %s", outs[i].name, outs[j].name);
    }
    if (g->ddelta.ptr && !a->delta.ptr)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "ddelta without delta");
    if (g->ddelta_bias && !a->delta.ptr)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "ddelta_bias without delta");
    TTC_TRY(check_floats("dstate_out", g->dstate_out, true));
    TTC_TRY(check_floats("dA", g->dA, true));
    TTC_TRY(check_floats("ddelta_bias", g->ddelta_bias, true));
    TTC_TRY(check_floats("dstate", g->dstate, true));
    if (ranges_meet(g->dstate, state_bytes(a), a->state, state_bytes(a)) || ranges_meet(g->dstate, state_bytes(a), g->dstate_out, state_bytes(a)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dstate overlaps state or dstate_out");
    GradDev& p = o.g;
    p = GradDev{};
    p.f = to_dev(a, false);
    const bool packed = a->seq_offsets;
    p.dy = dev_rows(g->dy, a->seq_offsets);
    p.dq = dev_rows(g->dq, a->seq_offsets);
    p.dk = dev_rows(g->dk, a->seq_offsets);
    p.dv = dev_rows(g->dv, a->seq_offsets);
    p.ddelta = dev_rows(g->ddelta, a->seq_offsets);
    p.head_dy = a->dv;
    p.vec_dq = bytes_at_once(p.dq, a->dk);
    p.vec_dk = bytes_at_once(p.dk, a->dk);
    p.vec_dv = bytes_at_once(p.dv, a->dv);
    p.f.vec_state = a->dv % 8 == 0 && floats_by_16_bytes(a->state) && floats_by_16_bytes(g->dstate_out) && floats_by_16_bytes(g->dstate);
    p.dstate_out = g->dstate_out;
    p.dA = g->dA;
    p.dbias = g->ddelta_bias;
    p.dstate = g->dstate;
    p.resident = sm_count(device);
    p.want_l = g->ddelta.ptr || g->dA || g->ddelta_bias;
    p.want_q = p.want_l || g->dq.ptr;
    p.want_kv = p.want_l || g->dk.ptr || g->dv.ptr;
    Scratch s(ws);
    o.o.n = 0;
    align(p.f.seqs, a->groups, a->dk, p.f.q, p.f.head_q, o.o, s);
    align(p.f.seqs, a->groups, a->dk, p.f.k, p.f.head_k, o.o, s);
    align(p.f.seqs, a->heads, a->dv, p.f.v, p.f.head_v, o.o, s);
    align(p.f.seqs, a->heads, a->dv, p.dy, p.head_dy, o.o, s);
    // float16: a power of two goes with each image of a state, so that it is one walk's
    o.splits = a->dtype == TTC_BF16 ? padded(a->dv) / kCols : 1;
    States& q = o.q;
    q = States{};
    TTC_TRY(take_pieces(device, a, o.splits, padded(a->dv) / o.splits, p.f, q, 2, s));
    // Walks both ways side by side, where one way leaves SMs idle (of packed sequences, whose shorter walks end early, where it fills them once): <Z, S_0> takes a kernel of its own
    // then, which reads both images again; else the second walk reads the states of the first as it goes.  One after the other and side by side: 4 x 1024 tokens, 96 walks of 64 x 64
    // 135 and 139 us, 72 walks 115 and 104; 11 documents of 8191 tokens in all, 88 walks 134 and 106 us, 132 walks 163 and 144, 176 walks of 128 x 64 177 and 183.
    o.together = p.f.pieces * a->heads * o.splits <= (packed ? sm_count(device) : sm_count(device) / 2);
    if (p.f.chunks > INT32_MAX / (2 * a->heads))
        return fail(TTC_STATUS_UNSUPPORTED, "%lld chunks, %d heads", (long long)p.f.chunks, a->heads);
    if (packed) {
        p.f.piece_map = s.take<int2>(p.f.chunks);
        p.f.seq_first = s.take<int>(a->batch + 1);
    }
    const size_t each = (size_t)p.f.chunks * a->heads, image = (size_t)padded(a->dk) * padded(a->dv) * 2 * (p.terms = a->dtype == TTC_BF16 && p.want_l ? 3 : 2);
    p.image_S = s.take<char>(std::max(each * image, (size_t)1));     // (there even for no chunks: a walk without images is one for what a piece adds)
    p.image_Z = s.take<char>(std::max(each * image, (size_t)1));
    if (a->dtype == TTC_F16) {
        p.unit_S = s.take<float>(each);
        p.unit_Z = s.take<float>(each);
    }
    q.seq_first = p.f.seq_first;
    q.way[0].k = p.f.k, q.way[0].head_k = p.f.head_k;
    q.way[0].v = p.f.v, q.way[0].head_v = p.f.head_v;
    q.way[0].given = a->state;
    q.way[0].factor = 1.f;
    q.way[0].image = p.image_S;
    q.way[0].unit = p.unit_S;
    q.way[1].back = 1;                           // with queries for keys and dy for values
    q.way[1].k = p.f.q, q.way[1].head_k = p.f.head_q;
    q.way[1].v = p.dy, q.way[1].head_v = p.head_dy;
    q.way[1].given = p.dstate_out;
    q.way[1].last = p.dstate;
    q.way[1].factor = a->scale;
    q.way[1].image = p.image_Z;
    q.way[1].unit = p.unit_Z;
    q.way[0].terms = q.way[1].terms = p.terms;
    q.way[0].image_bytes = q.way[1].image_bytes = padded(a->dk) * padded(a->dv) * 2;
    if (p.want_l) {
        p.tokens = s.take<float>(5 * each * kChunk);
        p.across_of = o.together ? 1 : o.splits * kWalkWarps;
        p.across = s.take<float>(each * p.across_of);
        if (o.together) {
            p.whole = q.way[0].whole = s.take<float>(each);
        } else {
            q.way[1].other = p.image_S;
            q.way[1].other_unit = p.unit_S;
            q.way[1].across = p.across;
        }
        p.bridges = s.take<float>(2 * each);
        p.sums = s.take<float>(2 * each);
    }
    if (p.f.share > 1) {
        const size_t rows = (size_t)(packed ? a->tokens : a->batch * a->tokens) * a->heads * a->dk;
        if (g->dq.ptr)
            p.part_q = s.take<float>(rows);
        if (g->dk.ptr)
            p.part_k = s.take<float>(rows);
    }
    o.bytes = s.used;
    return TTC_OK;
}

} // namespace

namespace ttc {

int attention_device_error(int* value)
{
    TTC_CUDA(cudaMemcpyFromSymbol(value, umma::g_error, sizeof(*value)));
    return TTC_OK;
}

} // namespace ttc

extern "C" {

int64_t ttc_decay_attention_workspace(int32_t device, const ttc_decay_args* a)
{
    Plan o;
    TTC_TRY(plan_forward(device, a, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_decay_attention(int32_t device, const ttc_decay_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    Plan o;
    TTC_TRY(plan_forward(device, a, workspace, o));
    TTC_TRY(check_output(a, false));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const AttnDev& p = o.p;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (p.pieces == 0)
        return TTC_OK;
    const dim3 grid((unsigned)(p.pieces * p.heads * o.splits));
    Maps maps[2] = {};
    const bool is_bf16 = a->dtype == TTC_BF16;
    TTC_TRY(describe(maps[0].q, p.q, a->groups, a->dk, p.head_q, p.seqs, is_bf16));
    TTC_TRY(describe(maps[0].k, p.k, a->groups, a->dk, p.head_k, p.seqs, is_bf16));
    TTC_TRY(describe(maps[0].v, p.v, a->heads, a->dv, p.head_v, p.seqs, is_bf16));
    TTC_TRY(align_all(p.seqs, o.o, st));
    auto go = [&](auto t, auto kc) {
        using T = decltype(t);
        constexpr int DK = decltype(kc)::value;
        if (p.piece_state) {
            States q = o.q;
            q.way[0].k = p.k, q.way[0].head_k = p.head_k;
            q.way[0].v = p.v, q.way[0].head_v = p.head_v;
            q.way[0].given = p.state;
            q.way[0].factor = 1.f;
            TTC_TRY((piece_states<T, DK, kCols>(maps, p, q, 1, o.splits, st)));
        }
        constexpr int smem = WalkShape<T, DK>::SMEM;
        TTC_TRY((allow_smem(walk_kernel<T, DK>, smem)));
        return launch_early("decay attention", walk_kernel<T, DK>, grid, kWalkBlock, smem, 1, st, maps[0], p);
    };
    constexpr std::integral_constant<int, 64> small;
    constexpr std::integral_constant<int, 128> large;
    if (a->dtype == TTC_BF16)
        return a->dk > 64 ? go(bf16(), large) : go(bf16(), small);
    return a->dk > 64 ? go(__half(), large) : go(__half(), small);
}

int ttc_decay_attention_step(int32_t device, const ttc_decay_args* a, void* cuda_stream)
{
    TTC_TRY(check(a, true));
    TTC_TRY(check_output(a, true));
    if (!a->state_out && a->batch)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "state_out is null");
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (a->batch == 0)
        return TTC_OK;
    const AttnDev p = to_dev(a, true);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool wide = a->dv % 4 == 0 && floats_by_16_bytes(a->state_out);
    int lanes = 8;
    while (lanes < 32 && lanes * (wide ? 4 : 1) < a->dv)
        lanes *= 2;
    auto go = [&](auto t) {
        using T = decltype(t);
        const int cols = lanes * (wide ? 4 : 1);
        return launch_early("decay attention, one token", wide ? decay_step_kernel<T, 4> : decay_step_kernel<T, 1>,
                            dim3((unsigned)(a->batch * a->heads), (unsigned)((a->dv + cols - 1) / cols)), kStepThreads, 0, 1, st, p, lanes);
    };
    return a->dtype == TTC_BF16 ? go(bf16()) : go(__half());
}

int64_t ttc_decay_attention_grad_workspace(int32_t device, const ttc_decay_args* a, const ttc_decay_grads* g)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_decay_attention_grad(int32_t device, const ttc_decay_args* a, const ttc_decay_grads* g, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const GradDev& p = o.g;
    const AttnDev& f = p.f;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    TTC_TRY(map_pieces(f, kChunk, 0, f.chunks, st));
    Maps maps[2] = {};
    const bool is_bf16 = a->dtype == TTC_BF16;
    TTC_TRY(describe(maps[0].k, f.k, a->groups, a->dk, f.head_k, f.seqs, is_bf16));
    TTC_TRY(describe(maps[0].v, f.v, a->heads, a->dv, f.head_v, f.seqs, is_bf16));
    TTC_TRY(describe(maps[1].k, f.q, a->groups, a->dk, f.head_q, f.seqs, is_bf16));
    TTC_TRY(describe(maps[1].v, p.dy, a->heads, a->dv, p.head_dy, f.seqs, is_bf16));
    TTC_TRY(align_all(f.seqs, o.o, st));
    return by_widths(a, [&](auto t, auto kc, auto vc) {
        using T = decltype(t);
        constexpr int DK = decltype(kc)::value, DV = decltype(vc)::value;
        constexpr int COLS = std::is_same<T, bf16>::value ? kCols : DV;
        TTC_TRY((chunk_states<T, DK, COLS>(maps, f, o.q, o.splits, o.together, st)));
        if (f.chunks && (p.want_q || p.want_kv)) {
            constexpr int smem = GradShape<DK, DV>::SMEM;
            TTC_TRY((allow_smem(grad_kernel<T, DK, DV>, smem)));
            TTC_TRY((launch_early("gradients of decay attention", grad_kernel<T, DK, DV>, dim3((unsigned)(f.chunks * f.heads * (p.want_q && p.want_kv ? 2 : 1))), kGradThreads, smem,
                                  1, st, maps[0], maps[1], p)));
        }
        if (f.chunks && (p.part_q || p.part_k))
            TTC_TRY((launch_early("gradients of decay attention, groups", a->dk % 4 ? grad_group_kernel<T, 1> : grad_group_kernel<T, 4>, dim3((unsigned)f.chunks, 8, 2), kThreads, 0, 1,
                                  st, p)));
        if (p.want_l) {
            if (f.chunks && o.together)
                TTC_TRY((launch_early("gradients of decay attention, across chunks", grad_across_kernel<T>, dim3((unsigned)(f.chunks * f.heads)), kThreads, 0, 1, st, p, DK * DV * 2)));
            if (f.chunks)
                TTC_TRY((launch_early("gradients of decay attention, decays", grad_decay_kernel<T>, dim3((unsigned)f.chunks, (unsigned)((f.heads + 3) / 4)), 128, 0, 1, st, p)));
            if (p.dA || p.dbias)
                TTC_TRY((launch_early("gradients of decay attention, heads", grad_head_kernel, dim3((unsigned)f.heads, 2), kThreads, 0, 1, st, p)));
        }
        return (int)TTC_OK;
    });
}

} // extern "C"
