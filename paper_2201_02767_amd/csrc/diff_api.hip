// C ABI of the rotary positions and of differential attention: argument validation and the launches. Everything here
// runs on the host; validation finishes before the first launch, and nothing allocates, synchronises or copies.
#include <stddef.h>
#include <stdint.h>

#include "diff_attn.h"

using namespace qta;

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool dtype_ok(qta_dtype t) { return t == QTA_F32 || t == QTA_BF16; }
int dtype_size(qta_dtype t) { return t == QTA_BF16 ? 2 : 4; }

// Shapes of a differential attention call, and its strides unless `shapes_only` (a workspace query).
qta_status check_diff(const qta_diff_attn_args* a, bool shapes_only)
{
    if (!a) return QTA_ERR_INVALID;
    if (a->B <= 0 || a->heads <= 0 || a->kv_heads <= 0 || a->Nq <= 0 || a->Nk <= 0 || a->d <= 0) return QTA_ERR_INVALID;
    if (a->heads % a->kv_heads != 0 || !dtype_ok(a->dtype)) return QTA_ERR_INVALID;
    if (a->d != 32 && a->d != 64) return QTA_ERR_UNSUPPORTED;
    // rows of a key head and keys are int, with room for the tiles behind the last
    const long long R = static_cast<long long>(a->Nq) * (a->heads / a->kv_heads);
    if (R > (1LL << 26) || a->Nk > (1 << 28) || a->heads > (1 << 16) || a->B > (1 << 24)) return QTA_ERR_UNSUPPORTED;
    if (shapes_only) return QTA_OK;
    if (!(a->lam_dtype == QTA_F32 || (a->lam_dtype == QTA_BF16 && a->dtype == QTA_BF16))) return QTA_ERR_INVALID;
    if (!a->q || !a->k || !a->v || !a->lam) return QTA_ERR_INVALID;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16)) return QTA_ERR_INVALID;
    if (!aligned(a->lam, dtype_size(a->lam_dtype)) || !aligned(a->lens, 4) || !aligned(a->q_pos, 4)) return QTA_ERR_INVALID;
    const int size = dtype_size(a->dtype), piece = 16 / size;
    const int64_t tokens[9] = {a->q_batch, a->q_token, a->q_head, a->k_batch, a->k_token, a->k_head, a->v_batch, a->v_token, a->v_head};
    for (const int64_t s : tokens)
        if (s < 0 || s % piece != 0) return QTA_ERR_INVALID;
    if (a->lam_batch < 0 || a->lam_token < 0 || a->lam_head < 0) return QTA_ERR_INVALID;
    // (the backward starts logits from the sums' logarithms over the scale)
    if (!(a->scale <= 0.f) && !(a->scale >= 0x1p-96f && a->scale <= 0x1p96f)) return QTA_ERR_INVALID;
    // inside one tile (at most 128 keys, or the rows of 65 queries) offsets are 31 bits
    const int64_t lim = (static_cast<int64_t>(1) << 30) / size;
    if (a->k_token > lim / 128 || a->v_token > lim / 128 || a->q_token > lim / 80 || a->q_head > lim / (2 * a->heads + 2)) return QTA_ERR_UNSUPPORTED;
    return QTA_OK;
}

DiffArgs make_args(const qta_diff_attn_args* a)
{
    DiffArgs x{};
    x.q = a->q;
    x.k = a->k;
    x.v = a->v;
    x.lam = a->lam;
    x.lam_bf16 = a->lam_dtype == QTA_BF16;
    x.causal = a->causal != 0;
    x.B = a->B;
    x.heads = a->heads;
    x.kv_heads = a->kv_heads;
    x.Nq = a->Nq;
    x.Nk = a->Nk;
    const int G = a->heads / a->kv_heads;
    x.R = a->Nq * G;
    x.div_G = make_fastdiv(G);
    x.qb = a->q_batch;
    x.qn = a->q_token;
    x.qh = a->q_head;
    x.kb = a->k_batch;
    x.kn = a->k_token;
    x.kh = a->k_head;
    x.vb = a->v_batch;
    x.vn = a->v_token;
    x.vh = a->v_head;
    x.lb = a->lam_batch;
    x.ln = a->lam_token;
    x.lh = a->lam_head;
    x.lens = a->lens;
    x.q_pos = a->q_pos;
    const float scale = a->scale > 0.f ? a->scale : 1.0f / sqrtf(static_cast<float>(a->d));
    x.scale = scale * 1.44269504088896f;
    return x;
}

// Regions of the forward's workspace.
struct FwdLayout {
    DiffParts parts;
    size_t part_sums, total;
};
FwdLayout fwd_layout(const qta_diff_attn_args* a)
{
    FwdLayout L{};
    const int R = a->Nq * (a->heads / a->kv_heads);
    L.parts = diff_key_parts(a->B, a->kv_heads, a->Nk, R, a->dtype == QTA_BF16);
    if (L.parts.splits == 1) return L;
    const size_t rows = static_cast<size_t>(L.parts.splits) * a->B * a->kv_heads * 2 * R;
    L.part_sums = align_up(rows * 2 * a->d * sizeof(float));
    L.total = L.part_sums + align_up(rows * 2 * sizeof(float));
    return L;
}

// Regions of the backward's workspace.
struct BwdLayout {
    size_t stats, dlam_rows, part, q_part, q_miss, total;
    int Rpad, splits, q_splits;
};
BwdLayout bwd_layout(const qta_diff_attn_args* a, bool lam_heads)
{
    BwdLayout L{};
    const int R = a->Nq * (a->heads / a->kv_heads);
    L.Rpad = (R + kDiffRowPad - 1) / kDiffRowPad * kDiffRowPad;
    size_t off = align_up(static_cast<size_t>(a->B) * a->kv_heads * kDiffStats * L.Rpad * sizeof(float));
    L.dlam_rows = off;
    if (lam_heads) off = align_up(off + static_cast<size_t>(a->B) * a->heads * a->Nq * sizeof(float));
    L.splits = diff_key_splits(a->B, a->kv_heads, a->Nk, R, a->causal != 0);
    L.part = off;
    if (L.splits > 1) off = align_up(off + static_cast<size_t>(L.splits) * a->B * a->Nk * a->kv_heads * 4 * a->d * sizeof(float));
    L.q_splits = diff_query_splits(a->B, a->kv_heads, a->Nk, R);
    if (L.q_splits > 1) {
        const size_t rows = static_cast<size_t>(L.q_splits) * a->B * a->kv_heads * R;
        L.q_part = off;
        off = align_up(off + rows * 2 * a->d * sizeof(float));
        L.q_miss = off;
        off = align_up(off + rows * sizeof(float));
    }
    L.total = off;
    return L;
}

// Whether every launch of a call is one that HIP takes.
bool fwd_fits(const qta_diff_attn_args* a, const FwdLayout& L)
{
    const long long groups = static_cast<long long>(a->B) * a->kv_heads, R = static_cast<long long>(a->Nq) * (a->heads / a->kv_heads);
    return diff_fwd_blocks(groups, R, L.parts) <= kDiffMaxBlocks && (L.parts.splits == 1 || diff_join_blocks(groups, R) <= kDiffMaxBlocks);
}
bool bwd_fits(const qta_diff_attn_args* a, const BwdLayout& L)
{
    const long long groups = static_cast<long long>(a->B) * a->kv_heads, R = static_cast<long long>(a->Nq) * (a->heads / a->kv_heads);
    return diff_dq_blocks(groups, R, L.q_splits) <= kDiffMaxBlocks && diff_dkv_blocks(groups, a->Nk, L.splits) + a->heads <= kDiffMaxBlocks &&
           (L.q_splits == 1 || diff_dq_join_blocks(groups, R, a->d) <= kDiffMaxBlocks) &&
           (L.splits == 1 || diff_dkv_join_blocks(groups, a->Nk, a->d, L.splits) <= kDiffMaxBlocks);
}

}  // namespace

extern "C" {

size_t qta_diff_attn_workspace_bytes(const qta_diff_attn_args* args)
{
    if (check_diff(args, true) != QTA_OK) return 0;
    const FwdLayout L = fwd_layout(args);
    if (!fwd_fits(args, L)) return 0;
    return L.total < kAlign ? kAlign : L.total;
}

qta_status qta_diff_attn(const qta_diff_attn_args* args, void* out, float* maps, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream)
{
    const qta_status st = check_diff(args, false);
    if (st != QTA_OK) return st;
    if (!out || !aligned(out, 16) || (maps != nullptr) != (lse != nullptr) || !aligned(maps, 16) || !aligned(lse, 4)) return QTA_ERR_INVALID;
    const FwdLayout L = fwd_layout(args);
    if (!fwd_fits(args, L)) return QTA_ERR_UNSUPPORTED;
    if (L.total > 0) {
        if (workspace_bytes < L.total) return QTA_ERR_WORKSPACE;
        if (!workspace || !aligned(workspace, kAlign)) return QTA_ERR_INVALID;
    }
    DiffArgs a = make_args(args);
    a.out = out;
    a.maps = maps;
    a.lse = lse;
    a.keys_apart = L.parts.keys_apart;
    a.splits = L.parts.splits;
    a.part = static_cast<float*>(workspace);
    a.part_sums = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + L.part_sums);
    return launch_diff_attn(a, args->d, args->dtype == QTA_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

size_t qta_diff_attn_backward_workspace_bytes(const qta_diff_attn_args* args)
{
    if (check_diff(args, true) != QTA_OK) return 0;
    const BwdLayout L = bwd_layout(args, true);
    return bwd_fits(args, L) ? L.total : 0;
}

qta_status qta_diff_attn_backward(const qta_diff_attn_args* args, const float* maps, const float* lse, const void* dout,
                                  void* dq, void* dk, void* dv, void* dlam, int dlam_heads, void* workspace,
                                  size_t workspace_bytes, void* stream)
{
    const qta_status st = check_diff(args, false);
    if (st != QTA_OK) return st;
    for (const void* p : {static_cast<const void*>(maps), dout, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
        if (!p || !aligned(p, 16)) return QTA_ERR_INVALID;
    if (!lse || !aligned(lse, 4) || !dlam || !aligned(dlam, dtype_size(args->lam_dtype))) return QTA_ERR_INVALID;
    if (!workspace || !aligned(workspace, kAlign)) return QTA_ERR_INVALID;
    const BwdLayout L = bwd_layout(args, dlam_heads != 0);
    if (!bwd_fits(args, L)) return QTA_ERR_UNSUPPORTED;
    if (workspace_bytes < L.total) return QTA_ERR_WORKSPACE;
    DiffBwdArgs a{};
    a.f = make_args(args);
    a.f.maps = const_cast<float*>(maps);
    a.f.lse = const_cast<float*>(lse);
    a.dout = dout;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    a.stats = reinterpret_cast<float*>(ws + L.stats);
    a.Rpad = L.Rpad;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.dlam = dlam;
    a.lam_heads = dlam_heads != 0;
    a.dlam_rows = reinterpret_cast<float*>(ws + L.dlam_rows);
    a.grad_scale = a.f.scale * kDiffLn2;
    a.splits = L.splits;
    a.part = reinterpret_cast<float*>(ws + L.part);
    a.q_splits = L.q_splits;
    a.q_part = reinterpret_cast<float*>(ws + L.q_part);
    a.q_miss = reinterpret_cast<float*>(ws + L.q_miss);
    return launch_diff_bwd(a, args->d, args->dtype == QTA_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

qta_status qta_rotary(const qta_rotary_tensor* tensors, int count, int B, int N, int d, int rot, int axes, int width,
                      int interleaved, int inverse, qta_dtype dtype, const double* freqs, const int32_t* pos,
                      int64_t pos_batch, int start, float scale, void* stream)
{
    if (!tensors || count < 1 || count > 2 || !freqs || !aligned(freqs, 8) || !aligned(pos, 4) || !dtype_ok(dtype)) return QTA_ERR_INVALID;
    if (B <= 0 || N <= 0 || d <= 0 || rot <= 0 || rot > d || (axes != 1 && axes != 2) || rot % (2 * axes) != 0) return QTA_ERR_INVALID;
    if (axes == 2 && !pos && (width <= 0 || N % width != 0 || start != 0)) return QTA_ERR_INVALID;
    if (pos_batch < 0) return QTA_ERR_INVALID;
    if (!pos && axes == 1 && (start > INT32_MAX - N || start < INT32_MIN + 1)) return QTA_ERR_INVALID;
    if (d > QTA_MAX_ROTARY_D || static_cast<int64_t>(B) * N > 0x7FFFFFFFLL) return QTA_ERR_UNSUPPORTED;
    RotaryArgs a{};
    int64_t heads = 0;
    for (int i = 0; i < count; ++i) {
        const qta_rotary_tensor& t = tensors[i];
        if (!t.x || !t.y || t.heads <= 0 || !aligned(t.x, dtype_size(dtype)) || !aligned(t.y, dtype_size(dtype))) return QTA_ERR_INVALID;
        for (const int64_t s : {t.x_batch, t.x_token, t.x_head, t.y_batch, t.y_token, t.y_head})
            if (s < 0) return QTA_ERR_INVALID;
        // in place: an element is written where it was read
        if (t.x == t.y && (t.x_batch != t.y_batch || t.x_token != t.y_token || t.x_head != t.y_head)) return QTA_ERR_INVALID;
        a.t[i] = RotaryTensor{t.x, t.y, t.heads, t.x_batch, t.x_token, t.x_head, t.y_batch, t.y_token, t.y_head};
        heads += t.heads;
    }
    if (heads > (1 << 16)) return QTA_ERR_UNSUPPORTED;
    // what one tensor's threads write is neither written nor read by the other's (further overlaps are the caller's to avoid)
    if (count == 2 && (tensors[0].y == tensors[1].y || tensors[0].y == tensors[1].x || tensors[0].x == tensors[1].y)) return QTA_ERR_INVALID;
    a.B = B;
    a.N = N;
    a.d = d;
    a.rot = rot;
    a.axes = axes;
    a.width = width;
    a.interleaved = interleaved != 0;
    a.inverse = inverse != 0;
    a.freqs = freqs;
    a.pos = pos;
    a.pos_b = pos_batch;
    a.start = start;
    a.scale = scale;
    return launch_rotary(a, dtype == QTA_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? QTA_OK : QTA_ERR_HIP;
}

}  // extern "C"
