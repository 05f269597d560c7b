// Host side of ttc_causal_conv, ttc_causal_conv_step and ttc_causal_conv_grad.
#include "block_host.h"
#include "causal_conv.cuh"

using namespace ttc;
using namespace ttc::blk;
using namespace ttc::conv;

namespace {

int check(const ttc_conv_args* a, bool step)
{
    if (!a)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "arguments are null");
    TTC_TRY(check_dtype(a->dtype, true));
    TTC_TRY(check_sequences(a->batch, step ? 1 : a->tokens, step ? nullptr : a->seq_offsets));
    if (a->d < 1)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "d = %d", a->d);
    if (a->taps < 2 || a->taps > 4)
        return fail(TTC_STATUS_UNSUPPORTED, "%d taps: 2 to 4 are served", a->taps);
    if (a->act != TTC_ACT_NONE && a->act != TTC_ACT_SILU)
        return fail(TTC_STATUS_UNSUPPORTED, "activation %d of a convolution", a->act);
    if ((a->d + kThreads - 1) / kThreads > kMaxGridY)
        return fail(TTC_STATUS_UNSUPPORTED, "d = %d", a->d);
    TTC_TRY(check_rows("x", a->x, a->dtype, step ? a->batch == 0 : a->tokens == 0 || a->batch == 0));
    TTC_TRY(check_floats("w", a->w, false));
    TTC_TRY(check_floats("bias", a->bias, true));
    TTC_TRY(check_floats("state", a->state, true, element_size(a->dtype)));
    return check_floats("state_out", a->state_out, true, element_size(a->dtype));
}

size_t window_bytes(const ttc_conv_args* a) { return (size_t)a->batch * (a->taps - 1) * a->d * element_size(a->dtype); }

// Channels that a thread takes, and whether every pointer and stride allows one access for them: else they are two, one by one.
struct Width {
    size_t size;
    int v;
    bool aligned;
    Width(int dtype, int d, int most) : size(element_size(dtype)), v(most), aligned(true) { fit(nullptr, d, 0); }
    void fit(const void* p, int64_t s0, int64_t s1)
    {
        while (aligned && (reinterpret_cast<uintptr_t>(p) % (v * size) || s0 % v || s1 % v)) {
            aligned = v > 2;
            v = 2;
        }
    }
    void rows(const ttc_rows& r, bool packed, bool step)
    {
        if (r.ptr)
            fit(r.ptr, packed ? 0 : r.bstride, step ? 0 : r.tstride);
    }
    void window(const void* p)
    {
        if (p)
            fit(p, 0, 0);
    }
};

ConvDev to_dev(const ttc_conv_args* a, bool step)
{
    ConvDev p = {};
    const int32_t* off = step ? nullptr : a->seq_offsets;
    p.seqs = Seqs{off, a->batch, step ? 1 : a->tokens};
    p.d = a->d;
    p.act = a->act;
    p.x = dev_rows(a->x, off);
    p.y = dev_rows(a->y, off);
    p.w = a->w;
    p.bias = a->bias;
    p.vec_w = reinterpret_cast<uintptr_t>(a->w) % 16 == 0;
    p.state = a->state;
    p.state_out = a->state_out;
    return p;
}

// Tokens of a tile: 128, or fewer (not below 16) while there are less than about six blocks for every SM.  A tile reads
// the W - 1 rows in front of it again.  (2 x 2048 x 4096: 19.3 us; with two blocks for every SM 25.6, with twelve 20.1.
// Gradients of 4 x 2048 x 4096: 62.8, 63.0 and 70.3.)
void set_tiles(ConvDev& p, int v, int sms)
{
    const int64_t cols = (p.d + (int64_t)v * kThreads - 1) / (v * kThreads);
    const int64_t seqs = p.seqs.offsets ? 1 : p.seqs.batch;
    p.tile = 128;
    while (p.tile > 16 && seqs * ((p.seqs.tokens + p.tile - 1) / p.tile) * cols < 6 * (int64_t)sms)
        p.tile /= 2;
    p.tiles = (p.seqs.tokens + p.tile - 1) / p.tile;
    p.all_tiles = seqs * p.tiles;
}

template <bool WIDE, typename F> int by_shape(int dtype, const Width& w, int taps, F&& f)
{
    return by_type(dtype, [&](auto t) {
        auto with = [&](auto vc, auto ac) {
            switch (taps) {
            case 2: return f(t, vc, ac, std::integral_constant<int, 2>());
            case 3: return f(t, vc, ac, std::integral_constant<int, 3>());
            default: return f(t, vc, ac, std::integral_constant<int, 4>());
            }
        };
        if constexpr (WIDE)
            if (w.v == 4)
                return with(std::integral_constant<int, 4>(), std::true_type());
        return w.aligned ? with(std::integral_constant<int, 2>(), std::true_type()) : with(std::integral_constant<int, 2>(), std::false_type());
    });
}

struct GradPlan {
    ConvDev p;
    Width w;
    size_t bytes;
    bool params;
    explicit GradPlan(const ttc_conv_args* a) : w(a ? a->dtype : TTC_F32, a ? a->d : 2, 2) {}
};

int plan_grad(int device, const ttc_conv_args* a, const ttc_conv_grads* g, void* ws, GradPlan& o)
{
    TTC_TRY(check(a, false));
    if (!g)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "gradients are null");
    TTC_TRY(check_rows("dy", g->dy, a->dtype, a->tokens == 0 || a->batch == 0));
    TTC_TRY(check_rows("dx", g->dx, a->dtype, true));
    TTC_TRY(check_floats("dw", g->dw, true));
    TTC_TRY(check_floats("dbias", g->dbias, true));
    TTC_TRY(check_floats("dstate", g->dstate, true, element_size(a->dtype)));
    TTC_TRY(check_floats("dstate_out", g->dstate_out, true, element_size(a->dtype)));
    const bool packed = a->seq_offsets;
    const size_t size = element_size(a->dtype);
    if (rows_overlap(g->dx, a->d, a->x, a->d, a->batch, a->tokens, packed, size) ||
        rows_overlap(g->dx, a->d, g->dy, a->d, a->batch, a->tokens, packed, size))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dx overlaps x or dy");
    const size_t bytes = window_bytes(a);
    if (ranges_meet(g->dstate, bytes, g->dstate_out, bytes) || ranges_meet(g->dstate, bytes, a->state, bytes))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dstate overlaps state or dstate_out");
    ConvDev& p = o.p;
    p = to_dev(a, false);
    p.dy = dev_rows(g->dy, a->seq_offsets);
    p.dx = dev_rows(g->dx, a->seq_offsets);
    p.dstate_out = g->dstate_out;
    p.dstate = g->dstate;
    p.dw = g->dw;
    p.dbias = g->dbias;
    Width& w = o.w;
    w.rows(a->x, packed, false);
    w.rows(g->dy, packed, false);
    w.rows(g->dx, packed, false);
    w.window(a->state);
    w.window(g->dstate);
    w.window(g->dstate_out);
    set_tiles(p, w.v, sm_count(device));
    o.params = g->dw || g->dbias;
    if (g->dstate && a->batch > 8 * (int64_t)(kMaxGridY - 8))
        return fail(TTC_STATUS_UNSUPPORTED, "gradients of %lld sequences", (long long)a->batch);
    Scratch s(ws);
    float* part = s.take<float>(o.params ? (size_t)p.all_tiles * (a->taps + 1) * a->d : 0);
    p.part = o.params ? part : nullptr;
    o.bytes = s.used;
    return TTC_OK;
}

} // namespace

extern "C" {

int ttc_causal_conv(int32_t device, const ttc_conv_args* a, void* cuda_stream)
{
    TTC_TRY(check(a, false));
    TTC_TRY(check_rows("y", a->y, a->dtype, a->tokens == 0 || a->batch == 0));
    const bool packed = a->seq_offsets;
    if (rows_overlap(a->y, a->d, a->x, a->d, a->batch, a->tokens, packed, element_size(a->dtype)))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "y overlaps x");
    const size_t bytes = window_bytes(a);
    const bool in_place = ranges_meet(a->state, bytes, a->state_out, bytes);
    if (in_place && a->state != a->state_out)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "state_out overlaps parts of state");
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (a->batch == 0)
        return TTC_OK;
    Width w(a->dtype, a->d, 2);
    w.rows(a->x, packed, false);
    w.rows(a->y, packed, false);
    w.window(a->state);
    ConvDev p = to_dev(a, false);
    set_tiles(p, w.v, sm_count(device));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return by_shape<false>(a->dtype, w, a->taps, [&](auto t, auto vc, auto ac, auto wc) {
        using T = decltype(t);
        constexpr int V = decltype(vc)::value, W = decltype(wc)::value;
        constexpr bool ALIGNED = decltype(ac)::value;
        const int64_t windows = a->state_out && !in_place ? a->batch : 0;
        if (p.all_tiles + windows) {
            const dim3 grid((unsigned)(p.all_tiles + windows), (a->d + V * kThreads - 1) / (V * kThreads));
            conv_kernel<T, V, ALIGNED, W><<<grid, kThreads, 0, st>>>(p);
            TTC_TRY(launched("causal convolution"));
        }
        if (in_place) {
            const dim3 grid((unsigned)a->batch, (a->d + kThreads - 1) / kThreads);
            TTC_TRY((launch_early("causal convolution, last windows", conv_window_kernel<T, W>, grid, kThreads, 0, 1, st, p)));
        }
        return TTC_OK;
    });
}

int ttc_causal_conv_step(int32_t device, const ttc_conv_args* a, void* cuda_stream)
{
    TTC_TRY(check(a, true));
    TTC_TRY(check_rows("y", a->y, a->dtype, a->batch == 0));
    if (!a->state_out && a->batch)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "state_out is null");
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (a->batch == 0)
        return TTC_OK;
    Width w(a->dtype, a->d, 4);
    w.rows(a->x, false, true);
    w.rows(a->y, false, true);
    w.window(a->state_out);
    // Narrower loads until every SM has many blocks (d = 4096: 64 sequences 2.7 us by four channels to a thread, 2.1 by two; 256
    // 5.5 and 5.3; 1024 16.2 and 17.8).
    if (w.v > 2 && a->batch * ((a->d + w.v * kThreads - 1) / (w.v * kThreads)) < 16 * (int64_t)sm_count(device))
        w.v = 2;
    const ConvDev p = to_dev(a, true);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return by_shape<true>(a->dtype, w, a->taps, [&](auto t, auto vc, auto ac, auto wc) {
        using T = decltype(t);
        constexpr int V = decltype(vc)::value, W = decltype(wc)::value;
        constexpr bool ALIGNED = decltype(ac)::value;
        const dim3 grid((unsigned)a->batch, (a->d + V * kThreads - 1) / (V * kThreads));
        return launch_early("causal convolution, one token", conv_step_kernel<T, V, ALIGNED, W>, grid, kThreads, 0, 1, st, p);
    });
}

int64_t ttc_causal_conv_grad_workspace(int32_t device, const ttc_conv_args* a, const ttc_conv_grads* g)
{
    GradPlan o(a);
    TTC_TRY(plan_grad(device, a, g, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_causal_conv_grad(int32_t device, const ttc_conv_args* a, const ttc_conv_grads* g, void* workspace,
                         int64_t workspace_bytes, void* cuda_stream)
{
    GradPlan o(a);
    TTC_TRY(plan_grad(device, a, g, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const ConvDev& p = o.p;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return by_shape<false>(a->dtype, o.w, a->taps, [&](auto t, auto vc, auto ac, auto wc) {
        using T = decltype(t);
        constexpr int V = decltype(vc)::value, W = decltype(wc)::value;
        constexpr bool ALIGNED = decltype(ac)::value;
        if (p.all_tiles) {
            const dim3 grid((unsigned)p.all_tiles, (a->d + V * kThreads - 1) / (V * kThreads));
            conv_grad_kernel<T, V, ALIGNED, W><<<grid, kThreads, 0, st>>>(p);
            TTC_TRY(launched("gradients of the causal convolution"));
        }
        // eight sequences to a block
        const int64_t empties = p.dstate && (a->seq_offsets || a->tokens == 0) ? (a->batch + 7) / 8 : 0;
        if (o.params || empties) {
            TTC_TRY((launch_early("gradients of the causal convolution, parameters", conv_param_kernel<T, W>,
                                  dim3((a->d + 31) / 32, (unsigned)(W + 1 + empties)), 256, 0, 1, st, p)));
        }
        return TTC_OK;
    });
}

} // extern "C"
