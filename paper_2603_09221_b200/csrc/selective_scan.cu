// Host side of ttc_selective_scan, ttc_selective_scan_step and ttc_selective_scan_grad.
#include <initializer_list>

#include "block_host.h"
#include "selective_scan_grad.cuh"

using namespace ttc;
using namespace ttc::blk;
using namespace ttc::sscan;

namespace {

int check(const ttc_scan_args* a, bool step)
{
    if (!a)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "arguments are null");
    TTC_TRY(check_dtype(a->dtype, true));
    TTC_TRY(check_sequences(a->batch, step ? 1 : a->tokens, step ? nullptr : a->seq_offsets));
    if (a->d < 1 || a->n < 1 || a->groups < 1 || a->d % a->groups)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "d = %d, n = %d, groups = %d", a->d, a->n, a->groups);
    if (a->n > 128)
        return fail(TTC_STATUS_UNSUPPORTED, "n = %d: 1 to 128 states are served", a->n);
    if (a->d > 4 * kMaxGridY || (int64_t)a->d * a->n > 128ll * kMaxGridY)
        return fail(TTC_STATUS_UNSUPPORTED, "d = %d, n = %d", a->d, a->n);
    const bool none = a->batch == 0 || (!step && a->tokens == 0);    // no rows, no addresses
    TTC_TRY(check_rows("x", a->x, a->dtype, none));
    TTC_TRY(check_rows("delta", a->delta, a->dtype, none));
    TTC_TRY(check_rows("B", a->B, a->dtype, none));
    TTC_TRY(check_rows("C", a->C, a->dtype, none));
    TTC_TRY(check_rows("z", a->z, a->dtype, true));
    TTC_TRY(check_floats("A", a->A, false));
    TTC_TRY(check_floats("D", a->D, true));
    TTC_TRY(check_floats("delta_bias", a->delta_bias, true));
    TTC_TRY(check_floats("state", a->state, true));
    return check_floats("state_out", a->state_out, true);
}

bool same_rows(const ttc_rows& a, const ttc_rows& b) { return a.ptr == b.ptr && a.tstride == b.tstride && a.bstride == b.bstride; }

size_t state_bytes(const ttc_scan_args* a) { return (size_t)a->batch * a->d * a->n * sizeof(float); }

int check_output(const ttc_scan_args* a, bool step)
{
    if (!step && a->state != a->state_out && ranges_meet(a->state, state_bytes(a), a->state_out, state_bytes(a)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "state_out overlaps parts of state");
    TTC_TRY(check_rows("y", a->y, a->dtype, a->batch == 0 || (!step && a->tokens == 0)));
    const int64_t tokens = step ? 1 : a->tokens, shared = (int64_t)a->groups * a->n;
    const bool packed = !step && a->seq_offsets;
    const size_t size = element_size(a->dtype);
    auto clash = [&](const ttc_rows& r, int64_t width) { return rows_overlap(a->y, a->d, r, width, a->batch, tokens, packed, size); };
    if ((clash(a->x, a->d) && !same_rows(a->y, a->x)) || (clash(a->z, a->d) && !same_rows(a->y, a->z)) ||
        clash(a->delta, a->d) || clash(a->B, shared) || clash(a->C, shared))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "y overlaps delta, B, C or parts of x or z");
    return TTC_OK;
}

int lanes_of(int n)
{
    int lanes = 2;
    while (lanes * 4 < n)
        lanes *= 2;
    return lanes;
}

template <typename F> int by_lanes(int lanes, F&& f)
{
    switch (lanes) {
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    default: return f(std::integral_constant<int, 32>());
    }
}

ScanDev to_dev(const ttc_scan_args* a, bool step, bool grad = false)
{
    ScanDev p = {};
    const int32_t* off = step ? nullptr : a->seq_offsets;
    p.seqs = Seqs{off, a->batch, step ? 1 : a->tokens};
    p.d = a->d;
    p.n = a->n;
    p.groups = a->groups;
    p.softplus = a->softplus;
    const int ch = grad ? 2 * kGradThreads / lanes_of(a->n) : channels_of(lanes_of(a->n));
    p.chan_blocks = (a->d / a->groups + ch - 1) / ch;
    p.x = dev_rows(a->x, off);
    p.delta = dev_rows(a->delta, off);
    p.B = dev_rows(a->B, off);
    p.C = dev_rows(a->C, off);
    p.z = dev_rows(a->z, off);
    p.y = dev_rows(a->y, off);
    p.A = a->A;
    p.D = a->D;
    p.delta_bias = a->delta_bias;
    p.state = a->state;
    p.state_out = a->state_out;
    p.pieces_per_seq = 1;
    return p;
}

struct Plan {
    ScanDev p;
    int64_t pieces;
    size_t bytes;
    bool pairs;
};

// Whether two neighbouring elements of every row can be accessed together: no pair may lie across two groups or past a row.
bool in_pairs(const ttc_scan_args* a, std::initializer_list<const ttc_rows*> rows)
{
    const size_t size = element_size(a->dtype);
    bool ok = a->d / a->groups % 2 == 0 && a->n % 2 == 0;
    for (const ttc_rows* r : rows)
        if (r->ptr)
            ok = ok && reinterpret_cast<uintptr_t>(r->ptr) % (2 * size) == 0 && r->tstride % 2 == 0 && (a->seq_offsets || r->bstride % 2 == 0);
    return ok;
}

// Pieces are counted in 32 bits, and are as many blocks.
int check_pieces(int64_t pieces)
{
    return pieces <= INT32_MAX ? (int)TTC_OK : fail(TTC_STATUS_UNSUPPORTED, "%lld pieces of sequences", (long long)pieces);
}

// Few sequences and channels leave SMs idle: then the tokens are cut into pieces, whose own shares of the state are found
// first (a second exponential per state and token) and handed on.  That pays where a sequence's work can be cut by three or more
// (2048 tokens, 1024 channels, 16 states, which are 16 blocks a sequence; in pieces and without: one sequence 39.9 and 148.7 us,
// four 115 and 151, six 155 and 152, eight 222 and 153); at the least, two pieces of 128 tokens, it costs nothing (22.1 and 21.2).
// Packed sequences are cut at their mean length: a longer one is worked on by several blocks, while the others' only piece has no
// share to find (1024 channels, one sequence of 4000 tokens and 40 of 100: 130 us against 349 uncut; 2048 channels, 16 of 500: 137
// against 127).
int plan_forward(int device, const ttc_scan_args* a, void* ws, Plan& o)
{
    TTC_TRY(check(a, false));
    ScanDev& p = o.p;
    p = to_dev(a, false);
    o.pieces = a->batch;
    o.pairs = in_pairs(a, {&a->x, &a->delta, &a->B, &a->C, &a->z, &a->y});
    o.bytes = 0;
    const int64_t sms = sm_count(device), columns = (int64_t)p.chan_blocks * a->groups;
    if (columns > kMaxGridY)
        return fail(TTC_STATUS_UNSUPPORTED, "d = %d, n = %d, groups = %d", a->d, a->n, a->groups);
    const int64_t rows = a->seq_offsets ? a->tokens : a->tokens * a->batch;
    int64_t want = 0;                            // pieces in all; two blocks of each SM hold all that are not more
    if (3 * a->batch * columns <= 2 * sms)
        want = 2 * sms / columns;
    else if (a->seq_offsets)
        want = a->batch;
    if (want && rows) {
        // (of equal sequences, as many to each)
        const int64_t each = a->seq_offsets ? 1 : want / a->batch;
        int64_t piece = ((a->seq_offsets ? (rows + want - 1) / want : (a->tokens + each - 1) / each) + 15) / 16 * 16;
        piece = piece < 128 ? 128 : piece;
        if (2 * piece <= a->tokens) {
            p.piece = piece;
            p.pieces_per_seq = (a->tokens + piece - 1) / piece;
            o.pieces = a->seq_offsets ? a->tokens / piece + a->batch : a->batch * p.pieces_per_seq;
            TTC_TRY(check_pieces(o.pieces));
            Scratch s(ws);
            if (a->seq_offsets) {
                p.piece_map = s.take<int2>(o.pieces);
                p.seq_first = s.take<int>(a->batch + 1);
            }
            p.local = s.take<float>((size_t)o.pieces * a->d * a->n);
            p.local_step = s.take<float>((size_t)o.pieces * a->d);
            o.bytes = s.used;
        }
    }
    return TTC_OK;
}

template <typename K> int allow_smem(K* kernel, size_t bytes)
{
    if (bytes > 48 * 1024)
        TTC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    return TTC_OK;
}

int map_pieces(const ScanDev& p, int64_t piece, int at_least, int64_t bound, cudaStream_t st)
{
    return launch_early("selective scan, pieces", piece_map_kernel, dim3(1), 1024, 0, 1, st, p.seqs, piece, at_least, bound,
                        const_cast<int2*>(p.piece_map), const_cast<int*>(p.seq_first));
}

struct GradPlan {
    GradDev g;
    size_t bytes;
    bool pairs;
};

int plan_grad(int device, const ttc_scan_args* a, const ttc_scan_grads* g, void* ws, GradPlan& o)
{
    TTC_TRY(check(a, false));
    if (!g)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "gradients are null");
    const struct { const char* name; const ttc_rows* r; int64_t width; } outs[] = {
        {"dx", &g->dx, a->d}, {"ddelta", &g->ddelta, a->d}, {"dz", &g->dz, a->d},
        {"dB", &g->dB, (int64_t)a->groups * a->n}, {"dC", &g->dC, (int64_t)a->groups * a->n}};
    const struct { const ttc_rows* r; int64_t width; } ins[] = {
        {&g->dy, a->d}, {&a->x, a->d}, {&a->delta, a->d}, {&a->z, a->d},
        {&a->B, (int64_t)a->groups * a->n}, {&a->C, (int64_t)a->groups * a->n}};
    TTC_TRY(check_rows("dy", g->dy, a->dtype, a->batch == 0 || a->tokens == 0));
    for (auto& out : outs) {
        TTC_TRY(check_rows(out.name, *out.r, a->dtype, true));
        for (auto& in : ins)
            if (rows_overlap(*out.r, out.width, *in.r, in.width, a->batch, a->tokens, a->seq_offsets, element_size(a->dtype)))
                return fail(TTC_STATUS_INVALID_ARGUMENT, "%s overlaps an input", out.name);
    }
    if (g->dz.ptr && !a->z.ptr)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dz without z");
    TTC_TRY(check_floats("dstate_out", g->dstate_out, true));
    TTC_TRY(check_floats("dA", g->dA, true));
    TTC_TRY(check_floats("dD", g->dD, true));
    TTC_TRY(check_floats("ddelta_bias", g->ddelta_bias, true));
    TTC_TRY(check_floats("dstate", g->dstate, true));
    if (ranges_meet(g->dstate, state_bytes(a), a->state, state_bytes(a)) || ranges_meet(g->dstate, state_bytes(a), g->dstate_out, state_bytes(a)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dstate overlaps state or dstate_out");
    GradDev& p = o.g;
    p = GradDev{};
    p.f = to_dev(a, false, true);
    const int64_t columns = (int64_t)p.f.chan_blocks * a->groups;
    if (columns > kMaxGridY)
        return fail(TTC_STATUS_UNSUPPORTED, "d = %d, n = %d, groups = %d", a->d, a->n, a->groups);
    p.dy = dev_rows(g->dy, a->seq_offsets);
    p.dx = dev_rows(g->dx, a->seq_offsets);
    p.ddelta = dev_rows(g->ddelta, a->seq_offsets);
    p.dB = dev_rows(g->dB, a->seq_offsets);
    p.dC = dev_rows(g->dC, a->seq_offsets);
    p.dz = dev_rows(g->dz, a->seq_offsets);
    p.dstate_out = g->dstate_out;
    p.dA = g->dA;
    p.dD = g->dD;
    p.ddelta_bias = g->ddelta_bias;
    p.dstate = g->dstate;
    o.pairs = in_pairs(a, {&a->x, &a->delta, &a->B, &a->C, &a->z, &g->dy, &g->dx, &g->ddelta, &g->dz});
    p.f.vec4 = a->n % 4 == 0;                    // the states' scratch begins on 256 bytes
    const int64_t run = kPiece * kRun, states = (int64_t)a->d * a->n;
    p.f.piece = run;
    p.f.pieces_per_seq = (a->tokens + run - 1) / run;
    p.runs = a->seq_offsets ? a->tokens / run + a->batch : a->batch * p.f.pieces_per_seq;
    TTC_TRY(check_pieces(p.runs));
    Scratch s(ws);
    if (a->seq_offsets) {
        p.f.piece_map = s.take<int2>(p.runs);
        p.f.seq_first = s.take<int>(a->batch + 1);
    }
    p.h = s.take<float>((size_t)p.runs * kRun * states);
    p.r = s.take<float>((size_t)p.runs * kRun * states);
    p.step = s.take<float>((size_t)p.runs * kRun * a->d);
    if (g->dA)
        p.part_A = s.take<float>((size_t)p.runs * states);
    if (g->dD || g->ddelta_bias)
        p.part_D = s.take<float>((size_t)p.runs * 2 * a->d);
    if (g->dB.ptr || g->dC.ptr)
        p.part_BC = s.take<float>((size_t)p.f.chan_blocks * p.runs * run * a->groups * 2 * lanes_of(a->n) * 4);
    o.bytes = s.used;
    return TTC_OK;
}

} // namespace

extern "C" {

int64_t ttc_selective_scan_workspace(int32_t device, const ttc_scan_args* a)
{
    Plan o;
    TTC_TRY(plan_forward(device, a, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_selective_scan(int32_t device, const ttc_scan_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    Plan o;
    TTC_TRY(plan_forward(device, a, workspace, o));
    TTC_TRY(check_output(a, false));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (o.pieces == 0)
        return TTC_OK;
    const ScanDev& p = o.p;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (p.piece_map)
        TTC_TRY(map_pieces(p, p.piece, 1, o.pieces, st));
    return by_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        return by_lanes(lanes_of(a->n), [&](auto lc) {
            constexpr int LANES = decltype(lc)::value;
            const dim3 grid((unsigned)o.pieces, (unsigned)(p.chan_blocks * p.groups));
            auto go = [&](auto vc) {
                constexpr int V = decltype(vc)::value;
                if (p.piece) {
                    constexpr size_t smem = Shape<LANES>::smem(true);
                    TTC_TRY(allow_smem(scan_kernel<T, LANES, true, V>, smem));
                    scan_kernel<T, LANES, true, V><<<grid, kThreads, smem, st>>>(p);
                    TTC_TRY(launched("selective scan, shares of the pieces"));
                }
                constexpr size_t smem = Shape<LANES>::smem(false);
                TTC_TRY(allow_smem(scan_kernel<T, LANES, false, V>, smem));
                scan_kernel<T, LANES, false, V><<<grid, kThreads, smem, st>>>(p);
                return launched("selective scan");
            };
            return o.pairs ? go(std::integral_constant<int, 2>()) : go(std::integral_constant<int, 1>());
        });
    });
}

int ttc_selective_scan_step(int32_t device, const ttc_scan_args* a, void* cuda_stream)
{
    TTC_TRY(check(a, true));
    TTC_TRY(check_output(a, true));
    if (!a->state_out && a->batch)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "state_out is null");
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (a->batch == 0)
        return TTC_OK;
    ScanDev p = to_dev(a, true);
    p.vec4 = a->n % 4 == 0 && reinterpret_cast<uintptr_t>(a->state_out) % 16 == 0 && reinterpret_cast<uintptr_t>(a->A) % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return by_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        return by_lanes(lanes_of(a->n), [&](auto lc) {
            constexpr int LANES = decltype(lc)::value, CH = kStepThreads / LANES;
            return launch_early("selective scan, one token", scan_step_kernel<T, LANES>, dim3((unsigned)a->batch, (a->d + CH - 1) / CH), kStepThreads, 0, 1, st, p);
        });
    });
}

int64_t ttc_selective_scan_grad_workspace(int32_t device, const ttc_scan_args* a, const ttc_scan_grads* g)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_selective_scan_grad(int32_t device, const ttc_scan_args* a, const ttc_scan_grads* g, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const GradDev& p = o.g;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (p.f.piece_map)
        TTC_TRY(map_pieces(p.f, p.f.piece, 0, p.runs, st));
    const int64_t states = (int64_t)a->d * a->n;
    return by_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        return by_lanes(lanes_of(a->n), [&](auto lc) {
            constexpr int LANES = decltype(lc)::value;
            using S = Tile<LANES>;
            const dim3 grid((unsigned)p.runs, (unsigned)(p.f.chan_blocks * p.f.groups));
            auto local = [&](auto vc) {
                constexpr int V = decltype(vc)::value;
                TTC_TRY(allow_smem(grad_local_kernel<T, LANES, V>, S::smem_local()));
                grad_local_kernel<T, LANES, V><<<grid, kGradThreads, S::smem_local(), st>>>(p);
                return launched("gradients of the selective scan, shares of the pieces");
            };
            auto pieces = [&](auto vc) {
                constexpr int V = decltype(vc)::value;
                TTC_TRY(allow_smem(grad_piece_kernel<T, LANES, V>, S::smem_piece()));
                grad_piece_kernel<T, LANES, V><<<grid, kGradThreads, S::smem_piece(), st>>>(p);
                return launched("gradients of the selective scan");
            };
            constexpr std::integral_constant<int, 2> two;
            constexpr std::integral_constant<int, 1> one;
            if (p.runs)
                TTC_TRY(o.pairs ? local(two) : local(one));
            if (a->batch) {
                const int v = a->n % 4 == 0 ? 4 : 1;
                TTC_TRY(launch_early("gradients of the selective scan, states and co-states", v == 4 ? grad_join_kernel<4> : grad_join_kernel<1>,
                                     dim3((unsigned)a->batch, (unsigned)((states / v + 127) / 128), 2), 128, 0, 1, st, p));
            }
            if (p.runs)
                TTC_TRY(o.pairs ? pieces(two) : pieces(one));
            const int64_t blocks = (p.dA ? (states + 31) / 32 : 0) + (p.dD || p.ddelta_bias ? 2 * (((int64_t)a->d + 31) / 32) : 0);
            if (blocks) {
                TTC_TRY((launch_early("gradients of the selective scan, parameters", grad_sum_kernel, dim3((unsigned)blocks), 256, 0, 1, st, p)));
            }
            if (p.part_BC && p.runs) {
                TTC_TRY((launch_early("gradients of the selective scan, B and C", grad_rows_kernel<T>, dim3((unsigned)p.runs, 4), 256, 0, 1, st, p, LANES * 4)));
            }
            return (int)TTC_OK;
        });
    });
}

} // extern "C"
