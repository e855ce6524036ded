// C ABI of group norm: argument validation and the launches. Everything here runs on the host; validation finishes before the
// first launch, and nothing allocates, synchronises or copies.
#include <stddef.h>
#include <stdint.h>

#include "group_norm.h"

using namespace qta;

namespace {

constexpr size_t kAlign = 256;
bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

qta_status check_norm(const qta_group_norm_args* a, bool shapes_only)
{
    if (!a) return QTA_ERR_INVALID;
    if (a->B <= 0 || a->N <= 0 || a->C <= 0 || a->groups <= 0 || a->C % a->groups != 0) return QTA_ERR_INVALID;
    if (a->dtype != QTA_F32 && a->dtype != QTA_BF16) return QTA_ERR_INVALID;
    if (a->C > (1 << 20) || static_cast<long long>(a->B) * a->N > (1LL << 30) || static_cast<long long>(a->B) * a->C > (1LL << 30)) return QTA_ERR_UNSUPPORTED;
    if (shapes_only) return QTA_OK;
    if (!(a->param_dtype == QTA_F32 || (a->param_dtype == QTA_BF16 && a->dtype == QTA_BF16))) return QTA_ERR_INVALID;
    if (a->act < QTA_ACT_NONE || a->act > QTA_ACT_GELU || !(a->eps >= 0.f)) return QTA_ERR_INVALID;
    const unsigned psize = a->param_dtype == QTA_BF16 ? 2 : 4;
    if (!a->x || !aligned(a->x, a->dtype == QTA_BF16 ? 2 : 4) || !aligned(a->weight, psize) || !aligned(a->bias, psize)) return QTA_ERR_INVALID;
    if (a->x_batch < 0 || a->x_token < 0) return QTA_ERR_INVALID;
    return QTA_OK;
}

bool use_bf16(const qta_group_norm_args* a) { return a->dtype == QTA_BF16; }
NormPlan plan(const qta_group_norm_args* a, int align, bool back)
{
    return norm_plan(a->B, a->N, a->C, a->groups, a->per_token != 0, use_bf16(a), align, back);
}
// Elements of the widest access that all addresses and strides allow.
int widest(const qta_group_norm_args* a, const void* p, const void* q, const void* r)
{
    const unsigned size = use_bf16(a) ? 2 : 4;
    int V = 16 / static_cast<int>(size);
    auto ok = [&](int v) {
        for (const void* x : {a->x, p, q, r})
            if (!aligned(x, v * size)) return false;
        return (a->B == 1 || a->x_batch % v == 0) && (a->N == 1 || a->x_token % v == 0);
    };
    while (V > 1 && !ok(V)) V /= 2;
    return V;
}
// The most that a call asks for, whatever its alignment: above kAlign, which says that a call takes none, unless it does.
size_t most_bytes(const qta_group_norm_args* a, bool back)
{
    size_t n = a->per_token && !back ? kAlign : 2 * kAlign;
    for (int v = use_bf16(a) ? 8 : 4; v >= 1; v /= 2) n = std::max(n, plan(a, v, back).bytes);
    return n;
}
bool fits(const qta_group_norm_args* a, const NormPlan& p)
{
    if (p.tokens) return p.blocks <= 65535;
    return static_cast<long long>(a->B) * p.slabs * p.blocks + a->C / 16 + 1 < (1LL << 32) / kNormThreads;
}
bool all_fit(const qta_group_norm_args* a, bool back)
{
    for (int v = use_bf16(a) ? 8 : 4; v >= 1; v /= 2)
        if (!fits(a, plan(a, v, back))) return false;
    return true;
}

NormArgs make_args(const qta_group_norm_args* a)
{
    NormArgs x{};
    x.x = a->x;
    x.weight = a->weight;
    x.bias = a->bias;
    x.param_bf16 = a->param_dtype == QTA_BF16;
    x.B = a->B;
    x.N = a->N;
    x.C = a->C;
    x.groups = a->groups;
    x.P = a->C / a->groups;
    x.xb = a->x_batch;
    x.xn = a->x_token;
    x.act = a->act;
    x.eps = a->eps;
    return x;
}

}  // namespace

extern "C" {

size_t qta_group_norm_workspace_bytes(const qta_group_norm_args* args)
{
    return check_norm(args, true) == QTA_OK && all_fit(args, false) ? most_bytes(args, false) : 0;
}

qta_status qta_group_norm(const qta_group_norm_args* args, void* y, float* stats, void* workspace, size_t workspace_bytes, void* stream)
{
    const qta_status st = check_norm(args, false);
    if (st != QTA_OK) return st;
    if (!y || y == args->x || !aligned(y, use_bf16(args) ? 2 : 4) || !aligned(stats, 8)) return QTA_ERR_INVALID;
    if (!all_fit(args, false)) return QTA_ERR_UNSUPPORTED;
    const NormPlan p = plan(args, widest(args, y, nullptr, nullptr), false);
    if (!p.tokens) {
        if (workspace_bytes < p.bytes) return QTA_ERR_WORKSPACE;
        if (!workspace || !aligned(workspace, kAlign)) return QTA_ERR_INVALID;
    }
    NormArgs a = make_args(args);
    a.y = y;
    a.stats = args->per_token ? nullptr : stats;
    a.part = static_cast<float*>(workspace);
    return launch_norm_forward(a, p, use_bf16(args), static_cast<hipStream_t>(stream)) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

size_t qta_group_norm_backward_workspace_bytes(const qta_group_norm_args* args)
{
    return check_norm(args, true) == QTA_OK && all_fit(args, true) ? most_bytes(args, true) : 0;
}

qta_status qta_group_norm_backward(const qta_group_norm_args* args, const float* stats, const void* dy, void* dx, void* dweight, void* dbias,
                                   void* workspace, size_t workspace_bytes, void* stream)
{
    const qta_status st = check_norm(args, false);
    if (st != QTA_OK) return st;
    const unsigned size = use_bf16(args) ? 2 : 4, psize = args->param_dtype == QTA_BF16 ? 2 : 4;
    if (!dy || !dx || dx == args->x || dx == dy || !aligned(dy, size) || !aligned(dx, size)) return QTA_ERR_INVALID;
    if (!aligned(dweight, psize) || !aligned(dbias, psize)) return QTA_ERR_INVALID;
    if (!all_fit(args, true)) return QTA_ERR_UNSUPPORTED;
    const NormPlan p = plan(args, widest(args, dy, dx, nullptr), true);
    if (!args->per_token && (!stats || !aligned(stats, 8))) return QTA_ERR_INVALID;
    if (!p.tokens || dweight || dbias) {
        if (workspace_bytes < p.bytes) return QTA_ERR_WORKSPACE;
        if (!workspace || !aligned(workspace, kAlign)) return QTA_ERR_INVALID;
    }
    NormArgs a = make_args(args);
    a.stats = const_cast<float*>(stats);
    a.dy = dy;
    a.dx = dx;
    a.dweight = dweight;
    a.dbias = dbias;
    a.part = !p.tokens || dweight || dbias ? static_cast<float*>(workspace) : nullptr;
    return launch_norm_backward(a, p, use_bf16(args), static_cast<hipStream_t>(stream)) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

}  // extern "C"
