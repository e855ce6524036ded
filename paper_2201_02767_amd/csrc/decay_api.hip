// C ABI of linear attention with a decay: argument validation and the launches. Everything here runs on the host; validation
// finishes before the first launch, and nothing allocates, synchronises or copies.
#include <stddef.h>
#include <stdint.h>

#include "decay_attn.h"

using namespace qta;

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool size_ok(int d) { return d == 32 || d == 64 || d == 128; }

// Shapes of a call, and its pointers and strides unless `shapes_only` (a workspace query).
qta_status check_decay(const qta_decay_attn_args* a, bool shapes_only)
{
    if (!a) return QTA_ERR_INVALID;
    if (a->B <= 0 || a->heads <= 0 || a->N <= 0 || a->dk <= 0 || a->dv <= 0) return QTA_ERR_INVALID;
    if (a->dtype != QTA_F32 && a->dtype != QTA_BF16) return QTA_ERR_INVALID;
    if (!size_ok(a->dk) || !size_ok(a->dv)) return QTA_ERR_UNSUPPORTED;
    // (token counts are int, with room for a segment behind the last)
    if (a->N > (1 << 29) || a->heads > (1 << 16) || static_cast<long long>(a->B) * a->heads > (1LL << 24)) return QTA_ERR_UNSUPPORTED;
    if (shapes_only) return QTA_OK;
    if (!a->q || !a->k || !a->v || !a->log_decay) return QTA_ERR_INVALID;
    for (const void* p : {a->q, a->k, a->v, static_cast<const void*>(a->state)})
        if (!aligned(p, 16)) return QTA_ERR_INVALID;
    if (!aligned(a->log_decay, 4) || !aligned(a->lens, 4)) return QTA_ERR_INVALID;
    const int size = a->dtype == QTA_BF16 ? 2 : 4, piece = 16 / size;
    for (const int64_t s : {a->q_batch, a->q_token, a->q_head, a->k_batch, a->k_token, a->k_head, a->v_batch, a->v_token, a->v_head})
        if (s < 0 || s % piece != 0) return QTA_ERR_INVALID;
    if (!(a->scale <= 0.f) && !(a->scale >= 0x1p-64f && a->scale <= 0x1p64f)) return QTA_ERR_INVALID;
    // inside a chunk offsets are 31 bits
    const int64_t lim = (static_cast<int64_t>(1) << 30) / size / 64;
    if (a->q_token > lim || a->k_token > lim || a->v_token > lim) return QTA_ERR_UNSUPPORTED;
    return QTA_OK;
}

bool use_bf16(const qta_decay_attn_args* a) { return a->dtype == QTA_BF16; }
float scale_of(const qta_decay_attn_args* a) { return a->scale > 0.f ? a->scale : 1.0f / sqrtf(static_cast<float>(a->dk)); }
size_t part_bytes(const qta_decay_attn_args* a, int segs)
{
    return align_up(static_cast<size_t>(a->B) * a->heads * segs * a->dk * a->dv * sizeof(float));
}

// Segments and workspace of a forward and of a backward (whose launches have up to three roles, and two states).
DecaySegments fwd_segments(const qta_decay_attn_args* a)
{
    return a->N <= kDecayStepTokens ? DecaySegments{1, a->N} : decay_segments(a->B, a->heads, a->N, a->dv, 1, use_bf16(a));
}
DecaySegments bwd_segments(const qta_decay_attn_args* a) { return decay_segments(a->B, a->heads, a->N, std::min(a->dk, a->dv), 2, use_bf16(a)); }
size_t fwd_bytes(const qta_decay_attn_args* a)
{
    const int segs = fwd_segments(a).segs;
    return segs > 1 ? part_bytes(a, segs) : 0;
}
size_t bwd_bytes(const qta_decay_attn_args* a)
{
    const int segs = bwd_segments(a).segs;
    return segs > 1 ? 2 * part_bytes(a, segs) : 0;
}
// Whether every launch of a call is one that HIP takes, in workgroups of at most 256 threads.
bool fits(const qta_decay_attn_args* a, int roles, int segs, bool step)
{
    const long long rows = static_cast<long long>(a->B) * a->heads;
    const long long scan = segs > 1 ? rows * (a->dk * a->dv / 1024) : 0;
    return std::max(step ? rows * decay_step_slices(a->dv) : roles * rows * segs, scan) <= kDecayMaxBlocks;
}
bool fwd_fits(const qta_decay_attn_args* a) { return fits(a, 1, fwd_segments(a).segs, a->N <= kDecayStepTokens); }
bool bwd_fits(const qta_decay_attn_args* a) { return fits(a, 3, bwd_segments(a).segs, false); }

struct Operand {
    const void* x;
    long long b, n, h;
};
DecayRole make_role(const Operand& q, const Operand& k, const Operand& v)
{
    DecayRole r{};
    r.q = q.x, r.qb = q.b, r.qn = q.n, r.qh = q.h;
    r.k = k.x, r.kb = k.b, r.kn = k.n, r.kh = k.h;
    r.v = v.x, r.vb = v.b, r.vn = v.n, r.vh = v.h;
    r.f = r.u = 1.f;
    return r;
}
DecayArgs make_args(const qta_decay_attn_args* a, const DecaySegments& s)
{
    DecayArgs x{};
    x.B = a->B;
    x.heads = a->heads;
    x.N = a->N;
    x.segs = s.segs;
    x.seg = s.seg;
    x.log_decay = a->log_decay;
    x.lens = a->lens;
    x.scale = scale_of(a);
    return x;
}
DecayScanArgs make_scan(const DecayArgs& x, int cells)
{
    DecayScanArgs s{};
    s.part = x.part;
    s.B = x.B;
    s.heads = x.heads;
    s.N = x.N;
    s.segs = x.segs;
    s.seg = x.seg;
    s.cells = cells;
    s.log_decay = x.log_decay;
    s.lens = x.lens;
    return s;
}

}  // namespace

extern "C" {

size_t qta_decay_attn_workspace_bytes(const qta_decay_attn_args* args)
{
    if (check_decay(args, true) != QTA_OK || !fwd_fits(args)) return 0;
    return std::max(fwd_bytes(args), kAlign);
}

qta_status qta_decay_attn(const qta_decay_attn_args* args, void* out, float* state_out, void* workspace, size_t workspace_bytes,
                          void* stream)
{
    const qta_status st = check_decay(args, false);
    if (st != QTA_OK) return st;
    if (!out || !aligned(out, 16) || !aligned(state_out, 16)) return QTA_ERR_INVALID;
    const DecaySegments seg = fwd_segments(args);
    if (!fwd_fits(args)) return QTA_ERR_UNSUPPORTED;
    if (seg.segs > 1) {
        if (workspace_bytes < fwd_bytes(args)) return QTA_ERR_WORKSPACE;
        if (!workspace || !aligned(workspace, kAlign)) return QTA_ERR_INVALID;
    }
    const auto s = static_cast<hipStream_t>(stream);
    const bool bf = use_bf16(args);
    if (args->N <= kDecayStepTokens) {
        DecayStepArgs x{};
        x.q = args->q, x.qb = args->q_batch, x.qn = args->q_token, x.qh = args->q_head;
        x.k = args->k, x.kb = args->k_batch, x.kn = args->k_token, x.kh = args->k_head;
        x.v = args->v, x.vb = args->v_batch, x.vn = args->v_token, x.vh = args->v_head;
        x.out = out;
        x.state = args->state;
        x.last = state_out;
        x.B = args->B;
        x.heads = args->heads;
        x.N = args->N;
        x.log_decay = args->log_decay;
        x.lens = args->lens;
        x.scale = scale_of(args);
        return launch_decay_step(x, args->dk, args->dv, bf, s) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
    }
    DecayArgs a = make_args(args, seg);
    a.roles = 1;
    a.part = static_cast<float*>(workspace);
    DecayRole& r = a.role[0];
    r = make_role({args->q, args->q_batch, args->q_token, args->q_head}, {args->k, args->k_batch, args->k_token, args->k_head},
                  {args->v, args->v_batch, args->v_token, args->v_head});
    r.out = out;
    r.s_row = args->dv;
    r.s_col = 1;
    r.f = a.scale;
    if (seg.segs > 1) {
        if (launch_decay_states(a, args->dk, args->dv, bf, s) != hipSuccess) return QTA_ERR_HIP;
        DecayScanArgs scan = make_scan(a, args->dk * args->dv);
        scan.state[0] = args->state;
        scan.last[0] = state_out;
        if (launch_decay_scan(scan, 1, s) != hipSuccess) return QTA_ERR_HIP;
        r.state = a.part;
    } else {
        r.state = args->state;
        r.last = state_out;
    }
    return launch_decay_chunks(a, args->dk, args->dv, bf, s) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

size_t qta_decay_attn_backward_workspace_bytes(const qta_decay_attn_args* args)
{
    if (check_decay(args, true) != QTA_OK || !bwd_fits(args)) return 0;
    return std::max(bwd_bytes(args), kAlign);
}

qta_status qta_decay_attn_backward(const qta_decay_attn_args* args, const void* dout, const float* dstate_out, void* dq, void* dk,
                                   void* dv, float* dstate, void* workspace, size_t workspace_bytes, void* stream)
{
    const qta_status st = check_decay(args, false);
    if (st != QTA_OK) return st;
    for (const void* p : {dout, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
        if (!p || !aligned(p, 16)) return QTA_ERR_INVALID;
    if (!aligned(dstate_out, 16) || !aligned(dstate, 16) || (dstate && dstate == dstate_out)) return QTA_ERR_INVALID;
    const DecaySegments seg = bwd_segments(args);
    if (!bwd_fits(args)) return QTA_ERR_UNSUPPORTED;
    if (seg.segs > 1) {
        if (workspace_bytes < bwd_bytes(args)) return QTA_ERR_WORKSPACE;
        if (!workspace || !aligned(workspace, kAlign)) return QTA_ERR_INVALID;
    }
    const auto s = static_cast<hipStream_t>(stream);
    const bool bf = use_bf16(args);
    const int DK = args->dk, DV = args->dv;
    const Operand q{args->q, args->q_batch, args->q_token, args->q_head}, k{args->k, args->k_batch, args->k_token, args->k_head},
        v{args->v, args->v_batch, args->v_token, args->v_head},
        d{dout, static_cast<long long>(args->N) * args->heads * DV, static_cast<long long>(args->heads) * DV, DV};
    DecayArgs a = make_args(args, seg);
    const float* before = args->state;          // S and R, dk x dv each
    const float* behind = dstate_out;
    if (seg.segs > 1) {
        // S from keys and values, R with time running back from queries and the upstream gradient
        a.part = static_cast<float*>(workspace);
        a.roles = 2;
        a.role[0] = make_role(q, k, v);
        a.role[1] = make_role(k, q, d);
        a.role[1].back = true;
        a.role[1].u = a.scale;
        a.role[0].s_row = a.role[1].s_row = DV;
        a.role[0].s_col = a.role[1].s_col = 1;
        if (launch_decay_states(a, DK, DV, bf, s) != hipSuccess) return QTA_ERR_HIP;
        DecayScanArgs scan = make_scan(a, DK * DV);
        scan.state[0] = before;
        scan.state[1] = behind;
        scan.last[1] = dstate;
        if (launch_decay_scan(scan, 2, s) != hipSuccess) return QTA_ERR_HIP;
        before = a.part;
        behind = a.part + static_cast<size_t>(args->B) * args->heads * seg.segs * DK * DV;
    }
    DecayRole rq = make_role(d, v, k), rk = make_role(v, d, q), rv = make_role(k, q, d);
    rq.out = dq;
    rq.state = before;
    rq.f = a.scale;
    rk.out = dk;
    rv.out = dv;
    rk.state = rv.state = behind;
    rk.back = rv.back = true;
    rk.u = rv.u = a.scale;
    rq.s_row = rk.s_row = 1;
    rq.s_col = rk.s_col = DV;
    rv.s_row = DV;
    rv.s_col = 1;
    if (seg.segs == 1) rv.last = dstate;
    a.role[0] = rq;
    a.role[1] = rk;
    a.role[2] = rv;
    a.roles = DK == DV ? 3 : 2;
    if (launch_decay_chunks(a, DV, DK, bf, s) != hipSuccess) return QTA_ERR_HIP;
    if (DK == DV) return QTA_OK;
    a.role[0] = rv;
    a.roles = 1;
    return launch_decay_chunks(a, DK, DV, bf, s) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

}  // extern "C"
