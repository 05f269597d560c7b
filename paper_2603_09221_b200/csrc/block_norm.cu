// Host side of ttc_block_norm and ttc_block_norm_grad.
#include <algorithm>
#include <type_traits>

#include "block_host.h"
#include "block_norm.cuh"

using namespace ttc;
using namespace ttc::blk;
using namespace ttc::bnorm;

namespace {

constexpr int kMaxChannels = 16384;

struct Operand {
    const char* name;
    const void* ptr;
    int64_t ld;
};

int check_operand(const ttc_norm_args* a, const Operand& o)
{
    if (!o.ptr)
        return TTC_OK;
    if (reinterpret_cast<uintptr_t>(o.ptr) % element_size(a->dtype))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s is not aligned to its elements", o.name);
    if (o.ld < a->d && (a->rows > 1 || o.ld < 0))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "%s: rows of %lld elements, d = %d", o.name, (long long)o.ld, a->d);
    return TTC_OK;
}

bool changes(const ttc_norm_args* a) { return a->w_post || a->z || a->scale || a->residual; }

int check(const ttc_norm_args* a)
{
    if (!a)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "arguments are null");
    TTC_TRY(check_dtype(a->dtype, true));
    if (a->rows < 0 || a->d < 1 || a->groups < 1 || a->d % a->groups)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "rows = %lld, d = %d, groups = %d", (long long)a->rows, a->d, a->groups);
    if (a->rows > kMaxRows)
        return fail(TTC_STATUS_UNSUPPORTED, "more than %lld rows", (long long)kMaxRows);
    if (a->d > kMaxChannels)
        return fail(TTC_STATUS_UNSUPPORTED, "d = %d: up to %d channels are served", a->d, kMaxChannels);
    if (a->groups > 1 && !a->w_post)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "groups without w_post");
    if (!(a->eps >= 0.f && a->eps < 3.4e38f))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "eps is negative or not finite");
    if (!a->x && a->rows)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "x is null");
    const Operand in[] = {{"x", a->x, a->ldx}, {"z", a->z, a->ldz}, {"residual", a->residual, a->ldr}, {"h", a->h, a->ldh}, {"y", a->y, a->ldy}};
    for (auto& o : in)
        TTC_TRY(check_operand(a, o));
    TTC_TRY(check_floats("w_post", a->w_post, true));
    TTC_TRY(check_floats("scale", a->scale, true));
    return check_floats("w_pre", a->w_pre, true);
}

// An output may be an input only where it is said, and then the whole of it.
int check_overlap(const ttc_norm_args* a, const Operand& out, const Operand& in, bool may_be)
{
    const ttc_rows o = {const_cast<void*>(out.ptr), 0, out.ld}, i = {const_cast<void*>(in.ptr), 0, in.ld};
    if (!rows_overlap(o, a->d, i, a->d, 1, a->rows, true, element_size(a->dtype)) || (may_be && out.ptr == in.ptr && (out.ld == in.ld || a->rows == 1)))
        return TTC_OK;
    return fail(TTC_STATUS_INVALID_ARGUMENT, "%s overlaps %s%s", out.name, may_be ? "parts of " : "", in.name);
}

struct Way {
    int v, k, threads, rows_per_block;
    int mixed;                                   // how groups of channels lie
    size_t smem;
};

int ceil_pow2(int v)
{
    int r = 1;
    while (r < v)
        r *= 2;
    return r;
}

// Vectors of 16 bytes where every row and parameter can be accessed so; else single elements.  Then as many
// threads as give each at most `most` vectors, with more for rows that would need over 512 of them, in whole warps.
Way way_of(const ttc_norm_args* a, NormDev& p, std::initializer_list<Operand> rows, int most)
{
    const int v = 16 / (int)element_size(a->dtype);
    bool vec = a->d % v == 0;
    for (auto& o : rows)
        vec = vec && (!o.ptr || (reinterpret_cast<uintptr_t>(o.ptr) % 16 == 0 && (o.ld % v == 0 || a->rows <= 1)));
    for (const float* w : {a->w_post, a->scale, a->w_pre})
        vec = vec && reinterpret_cast<uintptr_t>(w) % 16 == 0;
    Way o;
    o.v = vec ? v : 1;
    const int vectors = a->d / o.v;
    int threads = ceil_pow2((vectors + most - 1) / most);
    threads = threads < 32 ? 32 : threads > 512 ? 512 : threads;
    if (vectors > 2 * threads)
        threads = vectors > 4096 ? 1024 : ceil_pow2((vectors + 3) / 4) < 32 ? 32 : ceil_pow2((vectors + 3) / 4);
    const int k = (vectors + threads - 1) / threads;
    o.k = k <= 1 ? 1 : k <= 2 ? 2 : k <= 4 ? 4 : 16;
    // (160 threads for 152 vectors instead of 256: gradients of 13541 x 1216 134 -> 91 us, of 14563 x 1152 86 -> 58)
    const int each = o.k == 16 ? k : o.k;
    o.threads = threads = std::min(threads, ((vectors + each - 1) / each + 31) / 32 * 32);
    o.rows_per_block = threads == 32 ? kRowsOfWarps : 1;
    const int size = a->d / a->groups, vectors_of_group = size / o.v;
    p.lanes = size % o.v == 0 && vectors_of_group <= 32 && !(vectors_of_group & (vectors_of_group - 1)) ? vectors_of_group : 0;
    o.mixed = a->groups == 1 || p.lanes ? kNear : size % o.v || o.v == 1 ? kAcross : kWhole;
    o.smem = o.mixed ? (size_t)o.rows_per_block * (a->d + a->groups) * sizeof(float) : 0;
    return o;
}

template <typename F> int by_way(int dtype, const Way& w, F&& f)
{
    return by_type(dtype, [&](auto t) {
        constexpr int V = 16 / sizeof(t);
        constexpr std::integral_constant<int, V> wide;
        constexpr std::integral_constant<int, 1> single;
        auto of = [&](auto v, auto k) {
            if constexpr (decltype(v)::value > 1)
                if (w.mixed == kWhole)
                    return f(t, v, k, std::integral_constant<int, kWhole>());
            return w.mixed ? f(t, v, k, std::integral_constant<int, kAcross>()) : f(t, v, k, std::integral_constant<int, kNear>());
        };
        auto by_k = [&](auto v) {
            switch (w.k) {
            case 1: return of(v, std::integral_constant<int, 1>());
            case 2: return of(v, std::integral_constant<int, 2>());
            default: return of(v, std::integral_constant<int, 4>());
            }
        };
        if (w.v > 1)
            return by_k(wide);
        return w.k == 16 ? of(single, std::integral_constant<int, 16>()) : by_k(single);
    });
}

// The most that a call asks for: gradients of 512 threads (a ring of 240 bytes each) in groups of one channel (4096 of them, 8 bytes each), 152 KB; rows of 16384 without a ring, 128 KB.  A
// kernel's limit is set to this by every call that needs it set, and never to less: what one thread sets has to serve another's launch.
constexpr int kMostShared = 160 * 1024;
template <typename K> int allow_smem(K* kernel, size_t bytes)
{
    if (bytes > 40 * 1024)
        TTC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared));
    return TTC_OK;
}

NormDev to_dev(const ttc_norm_args* a)
{
    NormDev p = {};
    p.rows = a->rows;
    p.d = a->d;
    p.groups = a->groups;
    p.size = a->d / a->groups;
    p.eps = a->eps;
    p.per_row = 1.f / a->d;
    p.per_group = 1.f / p.size;
    p.x = a->x, p.ldx = a->ldx;
    p.z = a->z, p.ldz = a->ldz;
    p.w_post = a->w_post;
    p.scale = a->scale;
    p.w_pre = a->w_pre;
    return p;
}

int launch(const char* what, void (*kernel)(const NormDev), dim3 grid, const Way& w, int sms, cudaStream_t st, const NormDev& p)
{
    TTC_TRY(allow_smem(kernel, w.smem));
    const dim3 block(w.threads, w.rows_per_block);
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = block;
    c.dynamicSmemBytes = w.smem;
    c.stream = st;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &early;
    c.numAttrs = (int)grid.x <= 2 * sms ? 1 : 0;                     // where the blocks are few
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, p);
    return e == cudaSuccess ? launched(what) : fail(TTC_STATUS_CUDA_ERROR, "%s: %s", what, cudaGetErrorString(e));
}

struct GradPlan {
    NormDev p;
    Way w;
    int blocks;
    size_t bytes;
};

int plan_grad(int device, const ttc_norm_args* a, const ttc_norm_grads* g, void* ws, GradPlan& o)
{
    TTC_TRY(check(a));
    if (!g)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "gradients are null");
    const Operand ins[] = {{"x", a->x, a->ldx}, {"z", a->z, a->ldz}, {"h", a->h, a->ldh}, {"dy", g->dy, g->lddy}, {"dh", g->dh, g->lddh}};
    const Operand outs[] = {{"dx", g->dx, g->lddx}, {"dz", g->dz, g->lddz}, {"dresidual", g->dresidual, g->lddr}};
    for (int i = 3; i < 5; ++i)
        TTC_TRY(check_operand(a, ins[i]));
    for (int i = 0; i < 3; ++i) {
        TTC_TRY(check_operand(a, outs[i]));
        for (int j = 0; j < 5; ++j)
            TTC_TRY(check_overlap(a, outs[i], ins[j], i == 2 && j == 4));
        for (int j = 0; j < i; ++j)
            TTC_TRY(check_overlap(a, outs[i], outs[j], false));
    }
    if (a->rows && a->w_pre && (!g->dy || (!a->h && (changes(a) || g->dresidual))))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "w_pre without dy or h");
    if (g->dy && !a->w_pre)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "dy without w_pre");
    if ((g->dz && !a->z) || (g->dw_post && !a->w_post) || (g->dscale && !a->scale) || (g->dw_pre && !a->w_pre))
        return fail(TTC_STATUS_INVALID_ARGUMENT, "the gradient of an operand that is missing");
    TTC_TRY(check_floats("dw_post", g->dw_post, true));
    TTC_TRY(check_floats("dscale", g->dscale, true));
    TTC_TRY(check_floats("dw_pre", g->dw_pre, true));
    NormDev& p = o.p;
    p = to_dev(a);
    p.h_in = a->h ? a->h : a->x;
    p.ldh = a->h ? a->ldh : a->ldx;
    p.dy = g->dy, p.lddy = g->lddy;
    p.dh = g->dh, p.lddh = g->lddh;
    p.dx = g->dx, p.lddx = g->lddx;
    p.dz = g->dz, p.lddz = g->lddz;
    p.dr = g->dresidual, p.lddr = g->lddr;
    p.dw_post = g->dw_post;
    p.dscale = g->dscale;
    p.dw_pre = g->dw_pre;
    o.w = way_of(a, p, {ins[0], ins[1], ins[2], ins[3], ins[4], outs[0], outs[1], outs[2]}, 1);
    if (o.w.v > 1 && o.w.k == 1)
        o.w.smem += (size_t)kAhead * 5 * o.w.threads * o.w.rows_per_block * 16;
    // as many workers as are resident by their registers
    const int resident = (o.w.k == 1 && o.w.v < 8 ? 768 : 512) / (o.w.threads * o.w.rows_per_block);
    const int64_t most = (int64_t)sm_count(device) * (resident > 1 ? resident : 1);
    const int64_t all = (a->rows + o.w.rows_per_block - 1) / o.w.rows_per_block;
    o.blocks = (int)(all < most ? all : most);
    p.workers = o.blocks * o.w.rows_per_block;
    Scratch s(ws);
    if (g->dw_post || g->dscale || g->dw_pre)
        p.parts = s.take<float>((size_t)p.workers * 3 * a->d);
    o.bytes = s.used;
    return TTC_OK;
}

} // namespace

extern "C" {

int ttc_block_norm(int32_t device, const ttc_norm_args* a, void* cuda_stream)
{
    TTC_TRY(check(a));
    if (a->rows && !a->h && !a->y)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "h and y are null");
    if ((a->y != nullptr) != (a->w_pre != nullptr) && a->rows)
        return fail(TTC_STATUS_INVALID_ARGUMENT, "y and w_pre come together");
    const Operand x = {"x", a->x, a->ldx}, z = {"z", a->z, a->ldz}, r = {"residual", a->residual, a->ldr}, h = {"h", a->h, a->ldh}, y = {"y", a->y, a->ldy};
    for (const Operand* out : {&h, &y}) {
        for (const Operand* in : {&x, &z, &r})
            TTC_TRY(check_overlap(a, *out, *in, true));
    }
    TTC_TRY(check_overlap(a, y, h, false));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    if (a->rows == 0)
        return TTC_OK;
    NormDev p = to_dev(a);
    p.r = a->residual, p.ldr = a->ldr;
    p.h = a->h, p.ldh = a->ldh;
    p.y = a->y, p.ldy = a->ldy;
    const Way w = way_of(a, p, {x, z, r, h, y}, 2);
    const dim3 grid((unsigned)((a->rows + w.rows_per_block - 1) / w.rows_per_block));
    return by_way(a->dtype, w, [&](auto t, auto v, auto k, auto m) {
        return launch("block norm", norm_kernel<decltype(t), decltype(v)::value, decltype(k)::value, decltype(m)::value>, grid, w, sm_count(device), static_cast<cudaStream_t>(cuda_stream), p);
    });
}

int64_t ttc_block_norm_grad_workspace(int32_t device, const ttc_norm_args* a, const ttc_norm_grads* g)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, nullptr, o));
    return (int64_t)o.bytes;
}

int ttc_block_norm_grad(int32_t device, const ttc_norm_args* a, const ttc_norm_grads* g, void* workspace, int64_t workspace_bytes, void* cuda_stream)
{
    GradPlan o;
    TTC_TRY(plan_grad(device, a, g, workspace, o));
    TTC_TRY(check_workspace(workspace, workspace_bytes, o.bytes));
    DeviceScope scope;
    TTC_TRY(scope.enter(device));
    const NormDev& p = o.p;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (o.blocks)
        TTC_TRY(by_way(a->dtype, o.w, [&](auto t, auto v, auto k, auto m) {
            return launch("gradients of the block norm", norm_grad_kernel<decltype(t), decltype(v)::value, decltype(k)::value, decltype(m)::value>, dim3(o.blocks), o.w, sm_count(device), st, p);
        }));
    if (p.dw_post || p.dscale || p.dw_pre)
        TTC_TRY((launch_early("gradients of the block norm, parameters", norm_sum_kernel, dim3((unsigned)((a->d + 31) / 32), 3), 32 * kRuns, 0, 1, st, p)));
    return TTC_OK;
}

} // extern "C"
