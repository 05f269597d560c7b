// Host side of ttc_decay_attention, ttc_decay_attention_step and ttc_decay_attention_grad.
#include <type_traits>

#include "block_host.h"
#include "decay_attention_grad.cuh"
#include "device_error.h"

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

// Whether rows of heads of `width` elements can be accessed by 16 bytes (8 elements).
bool by_16_bytes(const ttc_rows& r, int width, bool packed)
{
    return width % 8 == 0 && reinterpret_cast<uintptr_t>(r.ptr) % 16 == 0 && r.tstride % 8 == 0 && (packed || r.bstride % 8 == 0);
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
    p.vec_q = by_16_bytes(a->q, a->dk, off);
    p.vec_k = by_16_bytes(a->k, a->dk, off);
    p.vec_v = by_16_bytes(a->v, a->dv, off);
    p.vec_y = by_16_bytes(a->y, a->dv, off);
    p.vec_state = a->dv % 8 == 0 && floats_by_16_bytes(a->state) && floats_by_16_bytes(a->state_out);
    p.A = a->A;
    p.delta_bias = a->delta_bias;
    p.state = a->state;
    p.state_out = a->state_out;
    p.chunks_per_seq = (p.seqs.tokens + kChunk - 1) / kChunk;
    p.chunks = off ? p.seqs.tokens / kChunk + a->batch : a->batch * p.chunks_per_seq;
    return p;
}

// Scratch that the states of the chunks take, for `p` to keep.
int take_states(const ttc_decay_args* a, AttnDev& p, Scratch& s)
{
    if (p.chunks > INT32_MAX)
        return fail(TTC_STATUS_UNSUPPORTED, "%lld chunks", (long long)p.chunks);
    const size_t each = (size_t)p.chunks * a->heads, elements = (size_t)padded(a->dk) * padded(a->dv);
    if (a->seq_offsets) {
        p.piece_map = s.take<int2>(p.chunks);
        p.seq_first = s.take<int>(a->batch + 1);
    }
    p.added = s.take<float>(each * elements);
    p.whole = s.take<float>(each);
    if (a->dtype == TTC_F16) {
        p.most = s.take<float>(each);
        p.most_given = s.take<float>((size_t)a->batch * a->heads);
    }
    return TTC_OK;
}

struct Plan {
    AttnDev p;
    size_t bytes;
};

int plan_forward(const ttc_decay_args* a, void* ws, Plan& o)
{
    TTC_TRY(check(a, false));
    o.p = to_dev(a, false);
    Scratch s(ws);
    TTC_TRY(take_states(a, o.p, s));
    const size_t each = (size_t)o.p.chunks * a->heads;
    o.p.image = s.take<char>(each * padded(a->dk) * padded(a->dv) * 2);
    if (a->dtype == TTC_F16)
        o.p.unit = s.take<float>(each);
    o.bytes = s.used;
    return TTC_OK;
}

template <typename K> int allow_smem(K* kernel, int bytes)
{
    TTC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return TTC_OK;
}

int map_chunks(const AttnDev& p, cudaStream_t st)
{
    if (!p.piece_map)
        return TTC_OK;
    return launch_early("decay attention, chunks", piece_map_kernel, dim3(1), 1024, 0, 1, st, p.seqs, (long long)kChunk, 0, p.chunks,
                        const_cast<int2*>(p.piece_map), const_cast<int*>(p.seq_first));
}

// Images of the states in front of every chunk (BACK: of the gradients of those behind), and the last ones.
template <typename T, int DK, int DV, bool BACK, bool SPLIT>
int chunk_states(const AttnDev& p, const Rows& a, const Rows& b, int vec_a, int vec_b, float factor, char* image, const float* given, float* last, float* unit,
                 cudaStream_t st)
{
    const dim3 grid((unsigned)p.chunks, (unsigned)p.heads);
    if (p.chunks) {
        constexpr int smem = StateShape<T, DK, DV>::SMEM;
        TTC_TRY((allow_smem(chunk_state_kernel<T, DK, DV, BACK>, smem)));
        TTC_TRY((launch_early("decay attention, what the chunks add", chunk_state_kernel<T, DK, DV, BACK>, grid, kThreads, smem, 1, st, p, a, b, vec_a, vec_b, factor, given)));
    }
    if (p.seqs.batch && (p.chunks || last))
        TTC_TRY((launch_early("decay attention, states", state_scan_kernel<T, DK, DV, BACK, SPLIT>, dim3((unsigned)(p.seqs.batch * p.heads), DK * DV / 8 / kThreads), kThreads,
                              0, 1, st, p, (const float*)p.added, image, given, last, (const float*)p.most, unit)));
    return TTC_OK;
}

struct GradPlan {
    GradDev g;
    size_t bytes;
};

int plan_grad(const ttc_decay_args* a, const ttc_decay_grads* g, void* ws, GradPlan& o)
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
    p.vec_dy = by_16_bytes(g->dy, a->dv, packed);
    p.vec_dq = by_16_bytes(g->dq, a->dk, packed);
    p.vec_dk = by_16_bytes(g->dk, a->dk, packed);
    p.vec_dv = by_16_bytes(g->dv, a->dv, packed);
    p.f.vec_state = a->dv % 8 == 0 && floats_by_16_bytes(a->state) && floats_by_16_bytes(g->dstate_out) && floats_by_16_bytes(g->dstate);
    p.dstate_out = g->dstate_out;
    p.dA = g->dA;
    p.dbias = g->ddelta_bias;
    p.dstate = g->dstate;
    p.want_l = g->ddelta.ptr || g->dA || g->ddelta_bias;
    p.want_q = p.want_l || g->dq.ptr;
    p.want_kv = p.want_l || g->dk.ptr || g->dv.ptr;
    Scratch s(ws);
    TTC_TRY(take_states(a, p.f, s));
    const size_t each = (size_t)p.f.chunks * a->heads, image = (size_t)padded(a->dk) * padded(a->dv) * 4;
    p.image_S = s.take<char>(each * image);
    p.image_Z = s.take<char>(each * image);
    if (a->dtype == TTC_F16) {
        p.unit_S = s.take<float>(each);
        p.unit_Z = s.take<float>(each);
    }
    if (p.want_l) {
        p.tokens = s.take<float>(5 * each * kChunk);
        p.across = s.take<float>(each);
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

int64_t ttc_decay_attention_workspace(int32_t, const ttc_decay_args* a)
{
    Plan o;
    TTC_TRY(plan_forward(a, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_decay_attention(int32_t device, const ttc_decay_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    Plan o;
    TTC_TRY(plan_forward(a, workspace, o));
    TTC_TRY(check_output(a, false));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const AttnDev& p = o.p;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    TTC_TRY(map_chunks(p, st));
    return by_widths(a, [&](auto t, auto kc, auto vc) {
        using T = decltype(t);
        constexpr int DK = decltype(kc)::value, DV = decltype(vc)::value;
        TTC_TRY((chunk_states<T, DK, DV, false, false>(p, p.k, p.v, p.vec_k, p.vec_v, 1.f, p.image, p.state, p.state_out, p.unit, st)));
        if (p.chunks) {
            constexpr int smem = OutShape<DK, DV>::SMEM;
            TTC_TRY((allow_smem(chunk_out_kernel<T, DK, DV>, smem)));
            TTC_TRY((launch_early("decay attention", chunk_out_kernel<T, DK, DV>, dim3((unsigned)p.chunks, (unsigned)p.heads), kThreads, smem, 1, st, p)));
        }
        return (int)TTC_OK;
    });
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

int64_t ttc_decay_attention_grad_workspace(int32_t, const ttc_decay_args* a, const ttc_decay_grads* g)
{
    GradPlan o;
    TTC_TRY(plan_grad(a, g, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_decay_attention_grad(int32_t device, const ttc_decay_args* a, const ttc_decay_grads* g, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    GradPlan o;
    TTC_TRY(plan_grad(a, g, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const GradDev& p = o.g;
    const AttnDev& f = p.f;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    TTC_TRY(map_chunks(f, st));
    return by_widths(a, [&](auto t, auto kc, auto vc) {
        using T = decltype(t);
        constexpr int DK = decltype(kc)::value, DV = decltype(vc)::value;
        TTC_TRY((chunk_states<T, DK, DV, false, true>(f, f.k, f.v, f.vec_k, f.vec_v, 1.f, p.image_S, f.state, nullptr, p.unit_S, st)));
        TTC_TRY((chunk_states<T, DK, DV, true, true>(f, f.q, p.dy, f.vec_q, p.vec_dy, f.scale, p.image_Z, p.dstate_out, p.dstate, p.unit_Z, st)));
        const dim3 grid((unsigned)f.chunks, (unsigned)f.heads);
        constexpr int smem = GradShape<DK, DV>::SMEM;
        if (f.chunks && p.want_q) {
            TTC_TRY((allow_smem(grad_q_kernel<T, DK, DV>, smem)));
            TTC_TRY((launch_early("gradients of decay attention, q", grad_q_kernel<T, DK, DV>, grid, kThreads, smem, 1, st, p)));
        }
        if (f.chunks && p.want_kv) {
            TTC_TRY((allow_smem(grad_kv_kernel<T, DK, DV>, smem)));
            TTC_TRY((launch_early("gradients of decay attention, k and v", grad_kv_kernel<T, DK, DV>, grid, kThreads, smem, 1, st, p)));
        }
        if (f.chunks && (p.part_q || p.part_k))
            TTC_TRY((launch_early("gradients of decay attention, groups", grad_group_kernel<T>, dim3((unsigned)f.chunks, 16), kThreads, 0, 1, st, p)));
        if (p.want_l) {
            if (f.chunks)
                TTC_TRY((launch_early("gradients of decay attention, decays", grad_decay_kernel<T>, dim3((unsigned)f.chunks, (unsigned)((f.heads + 3) / 4)), 128, 0, 1, st, p)));
            if (p.dA || p.dbias)
                TTC_TRY((launch_early("gradients of decay attention, heads", grad_head_kernel, dim3((unsigned)f.heads, 2), kThreads, 0, 1, st, p)));
        }
        return (int)TTC_OK;
    });
}

} // extern "C"
