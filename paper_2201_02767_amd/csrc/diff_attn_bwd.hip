// Differential attention, backward (the mathematics of the tiles is in diff_attn.h).
//
// With D = dO V^T, t_m = dO . O_m (O_m = P_m V) and the weights made again from the stored sums:
//   dS_0 = P_0 (D - t_0),   dS_1 = -lambda P_1 (D - t_1),   dlambda = -t_1
//   dQ_m = scale dS_m K_m,  dK_m = scale dS_m^T Q_m,        dV = (P_0 - lambda P_1)^T dO
// Two passes: dQ, a wave taking 32 rows through the keys, which also leaves the rows' statistics for dK and dV, a wave
// taking 32 keys through the rows of every query head that shares them. D, and in the key pass V's weights, serve both
// maps, so here a wave holds both. Each result is summed in one order: no atomics, the same bits every run.
// The query pass has dO at hand for t_m, and a launch before it for the statistics has to read dO again: 28 us of 4096 rows,
// 2 x 16 heads of d = 64 in bf16, 19 in the query pass. Sums of dlambda by head run beside the keys for a launch of 4.5 us.
//
// D starts from -t_0 instead of zero, and in the key pass of bf16 inputs, where a statistic is needed for every register,
// Q K^T from -lse / scale: a weight is then one product and one power of two away. t_m comes from results whose weights were rounded;
// the rows of P_1 (D - t_1), which with the exact t_1 sum to zero, give what is missing, and dlambda is exact to fp32.
#include <atomic>
#include <type_traits>

#include "diff_attn.h"

namespace qta {
namespace {

using namespace diff;

constexpr int kThreads = kDiffThreads;

__device__ __forceinline__ void store_dlambda(const DiffBwdArgs& a, int b, int i, int h, float x)
{
    const long long row = static_cast<long long>(b) * a.f.Nq + i;
    if (a.lam_heads) a.dlam_rows[static_cast<long long>(h) * a.f.B * a.f.Nq + row] = x;
    else if (a.f.lam_bf16) Storage<bf16>::store1(a.dlam, row * a.f.heads + h, x);
    else Storage<float>::store1(a.dlam, row * a.f.heads + h, x);
}

// Whether the key pass starts Q K^T from -lse / scale (bf16), or from zero as fp32 inputs need: the sum would be rounded at the
// size of lse / scale (dK and dV of 4000 rows and 300 keys, d = 64: 1.2e-6 off, from zero 6.6e-7, a plain fp32 form 7e-7).
template <typename T>
__device__ __forceinline__ constexpr bool from_statistics() { return sizeof(T) == 2; }

__device__ __forceinline__ float frag_elem(const Frag<bf16>& f, int j) { return static_cast<float>(f.v[j]); }
__device__ __forceinline__ float frag_elem(const Frag<float>& f, int j) { return f.v[j]; }

// A weight for each head: its rows' gradients summed by one workgroup.
__device__ __forceinline__ void sum_dlambda(const DiffBwdArgs& a, int head, float* part)
{
    const long long n = static_cast<long long>(a.f.B) * a.f.Nq;
    const float* const p = a.dlam_rows + head * n;
    float s[4] = {};
    long long i = threadIdx.x;
    for (; i + 3 * kThreads < n; i += 4 * kThreads)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += p[i + j * kThreads];
    for (; i < n; i += kThreads) s[0] += p[i];
    const float t = wave_sum_fast((s[0] + s[1]) + (s[2] + s[3]));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x != 0) return;
    const float x = (part[0] + part[1]) + (part[2] + part[3]);
    if (a.f.lam_bf16) Storage<bf16>::store1(a.dlam, head, x);
    else Storage<float>::store1(a.dlam, head, x);
}

// ---- dQ ----

// With `q_splits` > 1 a workgroup takes one part of its rows' keys and writes fp32 sums to `q_part` and `q_miss` (the first
// part's with t_1).
template <typename T, int D, int BN>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void diff_dq_kernel(DiffBwdArgs a)
{
    using KT = Tile<T, D>;
    using VT = Tile<T, 2 * D>;
    constexpr int ES = sizeof(T), BM = 128;
    constexpr int kK = KT::bytes(BN), kStage = 2 * kK + VT::bytes(BN);
    extern __shared__ __align__(1024) unsigned char lds_raw[];
    lds_byte* const lds = (lds_byte*)lds_raw;
    const DiffArgs& f = a.f;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int tiles_n = (f.R + BM - 1) / BM;
    const int logical = xcd_remap(blockIdx.x, gridDim.x);
    const int work = logical / a.q_splits, split = logical - work * a.q_splits;
    const int bh = work / tiles_n, tile = tiles_n - 1 - (work - bh * tiles_n);     // the longest rows first
    const int b = bh / f.kv_heads, g = bh - b * f.kv_heads, G = f.heads / f.kv_heads;
    const int row0 = tile * BM, row1 = min(row0 + BM, f.R);
    const DiffRange range = diff_range(f, b);
    const int kend = range.limit(fast_div(row1 - 1, f.div_G)), kmask = range.limit(fast_div(row0, f.div_G));

    const int rr = row0 + wave * 32 + (lane & 31), r = min(rr, f.R - 1);
    const int qi = fast_div(r, f.div_G), h = g * G + r - qi * G, lim = range.limit(qi);
    const long long qat = range.read_as(qi, f.Nq);
    float miss = 0.f;                       // sum of P_1 (D - t_1)
    Frag<T> qf[2][D / 16], of[D / 8];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
            qf[m][s] = global_frag<T>(f.q, b * f.qb + qat * f.qn + (2 * h + m) * f.qh + 16 * s + 8 * half);
    const long long orow = ((static_cast<long long>(b) * f.Nq + qat) * f.heads + h) * (2 * D);
#pragma unroll
    for (int s = 0; s < D / 8; ++s) of[s] = global_frag<T>(a.dout, orow + 16 * s + 8 * half);
    // t_m, of this lane's half of the channels and then of both; the first part's workgroups leave what the key pass needs
    float t0 = 0.f, t1 = 0.f;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
        const f32x4* const o = reinterpret_cast<const f32x4*>(f.maps + 2 * orow + 16 * s + 8 * half);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x4 y = o[j], z = o[2 * D / 4 + j];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                t0 = fmaf(frag_elem(of[s], 4 * j + k), y[k], t0);
                t1 = fmaf(frag_elem(of[s], 4 * j + k), z[k], t1);
            }
        }
    }
    t0 += other_half(t0);
    t1 += other_half(t1);
    if (lim == 0) t0 = t1 = 0.f;            // (an element without a key has no row to read instead)
    const float lam = lim > 0 ? diff_lambda(f, b, qi, h) : 0.f, nlam = -lam, nt0 = -t0, t01 = t0 - t1;
    const float* const lse = f.lse + (static_cast<long long>(b) * f.heads + h) * 2 * f.Nq + qi;
    const float nlse0 = -lse[0], nlse1 = -lse[f.Nq];
    if (split == 0 && half == 0 && rr < a.Rpad) {
        const bool row = rr < f.R && lim > 0;
        const float unit = from_statistics<T>() ? 1.0f / f.scale : 1.0f, nsign = lam < 0.f ? 1.0f : -1.0f;
        const float x[kDiffStats] = {nlse0 * unit, (nlse1 + __builtin_amdgcn_logf(fabsf(lam))) * unit, nt0, nsign * t01, nsign};
        float* const st = a.stats + static_cast<size_t>(bh) * kDiffStats * a.Rpad + rr;
#pragma unroll
        for (int p = 0; p < kDiffStats; ++p) st[static_cast<size_t>(p) * a.Rpad] = row ? x[p] : 0.f;
    }
    f32x16 acc[2][D / 32];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) acc[m][c] = f32x16{};

    auto stage = [&](int k0, lds_byte* at) {
        const int last = kend - 1 - k0;
        const auto kmap0 = tiles::map_resource(byte_at(f.k, b * f.kb + k0 * f.kn + (2 * g) * f.kh, ES));
        const auto kmap1 = tiles::map_resource(byte_at(f.k, b * f.kb + k0 * f.kn + (2 * g + 1) * f.kh, ES));
        const auto vmap = tiles::map_resource(byte_at(f.v, b * f.vb + k0 * f.vn + g * f.vh, ES));
        const uint32_t kstep = static_cast<uint32_t>(f.kn) * ES, vstep = static_cast<uint32_t>(f.vn) * ES;
        auto koff = [&](int x) { return static_cast<uint32_t>(min(x, last)) * kstep; };
        auto voff = [&](int x) { return static_cast<uint32_t>(min(x, last)) * vstep; };
        KT::stage(at, kmap0, BN, wave, 4, lane, koff);
        KT::stage(at + kK, kmap1, BN, wave, 4, lane, koff);
        VT::stage(at + 2 * kK, vmap, BN, wave, 4, lane, voff);
    };

    const int wend = row0 + wave * 32 < f.R ? range.limit(fast_div(min(row0 + wave * 32 + 32, f.R) - 1, f.div_G)) : 0;
    const uint32_t krow = lds_address(lds) + KT::row_base(lane), kcol = lds_address(lds) + KT::col_base(lane),
                   vrow = lds_address(lds) + VT::row_base(lane);
    auto keys = [&](int k0, auto odd) {
        constexpr uint32_t k0t = odd.value * kStage, k1t = k0t + kK, vt = k0t + 2 * kK;
#pragma unroll
        for (int u = 0; u < BN / 32; ++u) {
            if (k0 + 32 * u >= wend) break;
            f32x16 s0{}, s1{}, dp;
#pragma unroll
            for (int e = 0; e < 16; ++e) dp[e] = nt0;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                s0 = mma(KT::row_frag(krow, k0t, 32 * u, c), qf[0][c], s0);
                s1 = mma(KT::row_frag(krow, k1t, 32 * u, c), qf[1][c], s1);
            }
#pragma unroll
            for (int c = 0; c < D / 8; ++c) dp = mma(VT::row_frag(vrow, vt, 32 * u, c), of[c], dp);
            float d0[16], d1[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                d0[e] = exp2_fast(fmaf(s0[e], f.scale, nlse0)) * dp[e];
                d1[e] = exp2_fast(fmaf(s1[e], f.scale, nlse1)) * (dp[e] + t01);
            }
            if (k0 + 32 * u + 32 > kmask) {
                branch_here();
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k0 + 32 * u + acc_row(e, half) >= lim) {
                        d0[e] = 0.f;
                        d1[e] = 0.f;
                    }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                miss += d1[e];
                d1[e] *= nlam;
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const Frag<T> f0 = pack_frag<T>(d0 + 8 * w), f1 = pack_frag<T>(d1 + 8 * w);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    acc[0][c] = mma(KT::col_frag(kcol, k0t, 32 * u + 16 * w, c), f0, acc[0][c]);
                    acc[1][c] = mma(KT::col_frag(kcol, k1t, 32 * u + 16 * w, c), f1, acc[1][c]);
                }
            }
        }
    };
    const int all = (kend + BN - 1) / BN;
    const int first = static_cast<int>(static_cast<long long>(all) * split / a.q_splits);
    const int end = static_cast<int>(static_cast<long long>(all) * (split + 1) / a.q_splits);
    if (first < end) stage(first * BN, lds);
    for (int t = first; t < end; t += 2) {
        tiles::wait_lds_loads();
        __syncthreads();
        if (t + 1 < end) stage((t + 1) * BN, lds + kStage);
        keys(t * BN, std::integral_constant<int, 0>{});
        if (t + 1 >= end) break;
        tiles::wait_lds_loads();
        __syncthreads();
        if (t + 2 < end) stage((t + 2) * BN, lds);
        keys((t + 1) * BN, std::integral_constant<int, 1>{});
    }
    miss += other_half(miss);
    if (rr >= f.R) return;
    if (a.q_splits > 1) {
        const long long at = (static_cast<long long>(split) * f.B * f.kv_heads + bh) * f.R + r;
        if (half == 0) a.q_miss[at] = split == 0 ? t1 + miss : miss;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    store4<float>(a.q_part, (2 * at + m) * D + 32 * c + acc_row(e, half), acc[m][c][e], acc[m][c][e + 1],
                                  acc[m][c][e + 2], acc[m][c][e + 3]);
        return;
    }
    if (half == 0) store_dlambda(a, b, qi, h, -(t1 + miss));
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                store4<T>(a.dq, ((static_cast<long long>(b) * f.Nq + qi) * 2 * f.heads + 2 * h + m) * D + 32 * c + acc_row(e, half),
                          acc[m][c][e] * a.grad_scale, acc[m][c][e + 1] * a.grad_scale, acc[m][c][e + 2] * a.grad_scale,
                          acc[m][c][e + 3] * a.grad_scale);
}

// The parts' sums, in their order: four channels of one row a thread.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_dq_join_kernel(DiffBwdArgs a)
{
    const DiffArgs& f = a.f;
    const long long item = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x, rows = static_cast<long long>(f.B) * f.kv_heads * f.R;
    const long long at = item / (D / 2);
    if (at >= rows) return;
    const int c = 4 * static_cast<int>(item - at * (D / 2));
    const int bh = static_cast<int>(at / f.R), r = static_cast<int>(at - static_cast<long long>(bh) * f.R), G = f.heads / f.kv_heads;
    const int b = bh / f.kv_heads, i = fast_div(r, f.div_G), h = (bh - b * f.kv_heads) * G + r - i * G;
    const f32x4* const p = reinterpret_cast<const f32x4*>(a.q_part) + item;
    f32x4 x = *p;
#pragma unroll 4
    for (int s = 1; s < a.q_splits; ++s) x += p[s * rows * (D / 2)];
    store4<T>(a.dq, ((static_cast<long long>(b) * f.Nq + i) * f.heads + h) * (2 * D) + c, x[0] * a.grad_scale, x[1] * a.grad_scale,
              x[2] * a.grad_scale, x[3] * a.grad_scale);
    if (c != 0) return;
    float miss = 0.f;
    for (int s = 0; s < a.q_splits; ++s) miss += a.q_miss[s * rows + at];
    store_dlambda(a, b, i, h, -miss);
}

// ---- dK, dV ----

// A wave takes 32 keys; K stays in its registers, V (whose 32 more would leave room for one wave a SIMD only) in LDS.
// With `splits` > 1 a workgroup takes one part of the rows that see its keys and writes fp32 sums to `part`.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void diff_dkv_kernel(DiffBwdArgs a)
{
    using QT = Tile<T, D>;
    using OT = Tile<T, 2 * D>;
    constexpr int ES = sizeof(T), BM = 32, BN = kDiffKeys;
    constexpr int kQ = QT::bytes(BM), kO = OT::bytes(BM), kStats = 1024, kStage = 2 * kQ + kO + kStats;
    extern __shared__ __align__(1024) unsigned char lds_raw[];
    lds_byte* const lds = (lds_byte*)lds_raw;
    lds_byte* const vt = lds + 2 * kStage;
    const DiffArgs& f = a.f;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    if (static_cast<int>(blockIdx.x) >= a.key_groups) {             // behind the key tiles: lambda's gradients, a head each
        sum_dlambda(a, static_cast<int>(blockIdx.x) - a.key_groups, reinterpret_cast<float*>(lds_raw));
        return;
    }
    const int tiles_n = (f.Nk + BN - 1) / BN;
    const int logical = xcd_remap(blockIdx.x, a.key_groups);
    const int bh = logical / (tiles_n * a.splits), rest = logical - bh * tiles_n * a.splits;
    const int tile = rest / a.splits, split = rest - tile * a.splits;      // the keys that most rows see first
    const int b = bh / f.kv_heads, g = bh - b * f.kv_heads, G = f.heads / f.kv_heads;
    const DiffRange range = diff_range(f, b);
    const int k0 = tile * BN, wk0 = k0 + wave * 32, key = wk0 + (lane & 31);

    f32x16 av[2 * D / 32], ak[2][D / 32];
#pragma unroll
    for (int c = 0; c < 2 * D / 32; ++c) av[c] = f32x16{};
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) ak[m][c] = f32x16{};

    // rows that see any of these keys: from the first query at or behind k0 on; this workgroup's tiles of them
    const int i0 = range.causal ? min(max(0, k0 - range.pos), f.Nq) : 0;
    const bool seen = k0 < range.len && i0 < f.Nq;
    const int rbeg = seen ? i0 * G / BM * BM : 0, all = seen ? (f.R - rbeg + BM - 1) / BM : 0;
    const int t0 = static_cast<int>(static_cast<long long>(all) * split / a.splits);
    const int t1 = static_cast<int>(static_cast<long long>(all) * (split + 1) / a.splits);

    if (t0 < t1) {
        // (keys behind the last that any query sees are read as that one; their weights are masked)
        const int last = range.limit(f.Nq - 1) - 1;
        const auto vmap = tiles::map_resource(byte_at(f.v, b * f.vb + k0 * f.vn + g * f.vh, ES));
        OT::stage(vt, vmap, BN, wave, 4, lane,
                  [&](int r) { return static_cast<uint32_t>(min(r, last - k0)) * (static_cast<uint32_t>(f.vn) * ES); });
        Frag<T> kf[2][D / 16];
        const long long kr = min(key, last);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
                kf[m][s] = global_frag<T>(f.k, b * f.kb + kr * f.kn + (2 * g + m) * f.kh + 16 * s + 8 * half);

        const auto smap = tiles::map_resource(reinterpret_cast<const unsigned char*>(a.stats + static_cast<size_t>(bh) * kDiffStats * a.Rpad));
        auto stage = [&](int r0, lds_byte* at) {
            const int i_first = fast_div(r0, f.div_G);
            const auto qmap0 = tiles::map_resource(byte_at(f.q, b * f.qb + i_first * f.qn + (2 * g * G) * f.qh, ES));
            const auto omap = tiles::map_resource(
                byte_at(a.dout, ((static_cast<long long>(b) * f.Nq + i_first) * f.heads + g * G) * (2 * D), ES));
            // (rows before the first that sees any of these keys are read as that one: they may hold anything)
            auto place = [&](int r, int* i, int* hh) {
                const int x = min(max(r0 + r, i0 * G), f.R - 1);
                *i = fast_div(x, f.div_G);
                *hh = x - *i * G;
                *i -= i_first;
            };
            auto qoff = [&](int r) {
                int i, hh;
                place(r, &i, &hh);
                return static_cast<uint32_t>((i * static_cast<int>(f.qn) + 2 * hh * static_cast<int>(f.qh)) * ES);
            };
            auto qoff1 = [&](int r) { return qoff(r) + static_cast<uint32_t>(f.qh) * ES; };
            auto ooff = [&](int r) {
                int i, hh;
                place(r, &i, &hh);
                return static_cast<uint32_t>((i * f.heads + hh) * (2 * D) * ES);
            };
            QT::stage(at, qmap0, BM, wave, 4, lane, qoff);
            QT::stage(at + kQ, qmap0, BM, wave, 4, lane, qoff1);
            OT::stage(at + 2 * kQ, omap, BM, wave, 4, lane, ooff);
            // five statistics of the 32 rows, 128 bytes each (lanes behind the fifth repeat it)
            if (wave == 0) {
                const int p = min(lane >> 3, kDiffStats - 1);
                tiles::load_lds16(smap, (static_cast<uint32_t>(p) * a.Rpad + r0 + 4 * (lane & 7)) * 4u, 0, at + 2 * kQ + kO);
            }
        };

        // the first row that sees this lane's key, and one that sees every key of the wave (R: none)
        auto first_row = [&](int x) { return x >= range.len ? f.R : range.causal ? min(max(0, x - range.pos), f.Nq) * G : 0; };
        const int see = first_row(key), wave_see = first_row(wk0 + 31);
        // (whole rows are added, so that the bases keep their bits below)
        const uint32_t base0 = lds_address(lds);
        uint32_t qrow = base0 + QT::row_base(lane), qcol = base0 + QT::col_base(lane), orow = base0 + OT::row_base(lane),
                 ocol = base0 + OT::col_base(lane), vrow = orow + 32 * wave * OT::kRow;
        uint32_t srow = base0 + 16 * half;
        // the 32 rows from r0 on; the bases are those of their stage, so that everything else is an immediate
        auto rows = [&](int r0) {
            constexpr uint32_t cur = 0, vw = 2 * kStage;
            opaque(qrow);
            opaque(qcol);
            opaque(orow);
            opaque(ocol);
            opaque(vrow);
            const bool edge = r0 < wave_see || r0 + BM > f.R;
            // four rows' statistics at a time: rows 8 (e / 4) + 4 half .. + 3
            constexpr uint32_t st = cur + 2 * kQ + kO;
            auto stat = [&](int plane, int e) { return *lds_at<f32x4>(srow + (st + plane * 128 + 8 * e)); };
            auto from = [&](int plane) {
                f32x16 x;
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 y = stat(plane, e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[e + j] = y[j];
                }
                return x;
            };
            f32x16 dp = from(2);
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                dp = mma(OT::row_frag(orow, cur + 2 * kQ, 0, c), OT::row_frag(vrow, vw, 0, c), dp);
                if (c % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
            float w[16];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                f32x16 s = from_statistics<T>() ? from(m) : f32x16{};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) s = mma(QT::row_frag(qrow, cur + m * kQ, 0, c), kf[m][c], s);
                float ds[16];
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    f32x4 t{}, sign{}, nlse{};
                    if constexpr (!from_statistics<T>()) nlse = stat(m, e);
                    if (m == 1) {
                        t = stat(3, e);
                        sign = stat(4, e);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = exp2_fast(from_statistics<T>() ? s[e + j] * f.scale : fmaf(s[e + j], f.scale, nlse[j]));
                        ds[e + j] = p * (m == 0 ? dp[e + j] : fmaf(sign[j], dp[e + j], t[j]));
                        w[e + j] = m == 0 ? p : fmaf(sign[j], p, w[e + j]);
                    }
                }
                if (edge) {
                    branch_here();
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int r = r0 + acc_row(e, half);
                        if (r < see || r >= f.R) ds[e] = w[e] = 0.f;
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const Frag<T> fd = pack_frag<T>(ds + 8 * u);
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) ak[m][c] = mma(QT::col_frag(qcol, cur + m * kQ, 16 * u, c), fd, ak[m][c]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const Frag<T> fw = pack_frag<T>(w + 8 * u);
#pragma unroll
                for (int c = 0; c < 2 * D / 32; ++c) av[c] = mma(OT::col_frag(ocol, cur + 2 * kQ, 16 * u, c), fw, av[c]);
            }
        };
        stage(rbeg + t0 * BM, lds);
        for (int t = t0; t < t1; ++t) {
            const bool odd = (t - t0) & 1;
            tiles::wait_lds_loads();
            __syncthreads();
            if (t + 1 < t1) stage(rbeg + (t + 1) * BM, odd ? lds : lds + kStage);
            rows(rbeg + t * BM);
            const uint32_t move = odd ? -kStage : kStage;
            qrow += move;
            qcol += move;
            orow += move;
            ocol += move;
            srow += move;
        }
    }
    if (key >= f.Nk) return;
    const long long krow = (static_cast<long long>(b) * f.Nk + key) * f.kv_heads + g;
    auto write = [&](auto type, void* dk, void* dv, long long at, int row, float scale) {
        using O = decltype(type);
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
                    store4<O>(dk, at * row + m * D + 32 * c + acc_row(e, half), ak[m][c][e] * scale, ak[m][c][e + 1] * scale,
                              ak[m][c][e + 2] * scale, ak[m][c][e + 3] * scale);
#pragma unroll
            for (int c = 0; c < 2 * D / 32; ++c)
                store4<O>(dv, at * row + 32 * c + acc_row(e, half), av[c][e], av[c][e + 1], av[c][e + 2], av[c][e + 3]);
        }
    };
    if (a.splits == 1) {
        write(T{}, a.dk, a.dv, krow, 2 * D, a.grad_scale);
    } else {
        // [split][key row][dK_0, dK_1, dV]
        const long long rows = static_cast<long long>(f.B) * f.Nk * f.kv_heads;
        write(float{}, a.part, a.part + 2 * D, split * rows + krow, 4 * D, 1.0f);
    }
}

// The parts' sums, in their order: four channels of one key by SLICES threads, each adding a run of the parts.
template <typename T, int D, int SLICES>
__global__ __launch_bounds__(kThreads) void diff_dkv_join_kernel(DiffBwdArgs a)
{
    constexpr int ITEMS = kThreads / SLICES;
    __shared__ f32x4 sums[SLICES == 1 ? 1 : kThreads];
    const int in = threadIdx.x % ITEMS, slice = threadIdx.x / ITEMS;
    const long long item = static_cast<long long>(blockIdx.x) * ITEMS + in;
    const long long total = static_cast<long long>(a.f.B) * a.f.Nk * a.f.kv_heads * D;
    const int first = a.splits * slice / SLICES, end = a.splits * (slice + 1) / SLICES;     // (never empty)
    f32x4 x{};
    if (item < total) {
        const f32x4* const p = reinterpret_cast<const f32x4*>(a.part) + item;
        x = p[first * total];
#pragma unroll 4
        for (int s = first + 1; s < end; ++s) x += p[s * total];
    }
    if constexpr (SLICES > 1) {
        sums[threadIdx.x] = x;
        __syncthreads();
        if (slice != 0) return;
#pragma unroll
        for (int s = 1; s < SLICES; ++s) x += sums[s * ITEMS + in];
    }
    if (item >= total) return;
    const long long row = item / D;
    const int c = 4 * static_cast<int>(item - row * D);
    if (c < 2 * D) store4<T>(a.dk, row * (2 * D) + c, x[0] * a.grad_scale, x[1] * a.grad_scale, x[2] * a.grad_scale, x[3] * a.grad_scale);
    else store4<T>(a.dv, row * (2 * D) + c - 2 * D, x[0], x[1], x[2], x[3]);
}

template <typename T, int D>
hipError_t launch_bwd(const DiffBwdArgs& args, hipStream_t stream)
{
    static std::atomic<unsigned long long> configured_q{0}, configured_k{0};
    constexpr int ES = static_cast<int>(sizeof(T)), BN = 32;
    DiffBwdArgs a = args;
    const long long bh = static_cast<long long>(a.f.B) * a.f.kv_heads;
    const long long qblocks = diff_dq_blocks(bh, a.f.R, a.q_splits), kblocks = diff_dkv_blocks(bh, a.f.Nk, a.splits);
    const long long heads = a.lam_heads ? a.f.heads : 0;
    a.key_groups = static_cast<int>(kblocks);
    hipError_t e = set_max_lds_once(reinterpret_cast<const void*>(&diff_dq_kernel<T, D, BN>), configured_q);
    if (e != hipSuccess) return e;
    e = set_max_lds_once(reinterpret_cast<const void*>(&diff_dkv_kernel<T, D>), configured_k);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((diff_dq_kernel<T, D, BN>), dim3(static_cast<unsigned>(qblocks)), dim3(kThreads), 2 * BN * 4 * D * ES,
                       stream, a);
    if (a.q_splits > 1)
        hipLaunchKernelGGL((diff_dq_join_kernel<T, D>), dim3(static_cast<unsigned>(diff_dq_join_blocks(bh, a.f.R, D))),
                           dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL((diff_dkv_kernel<T, D>), dim3(static_cast<unsigned>(kblocks + heads)), dim3(kThreads),
                       2 * (32 * 4 * D * ES + 1024) + kDiffKeys * 2 * D * ES, stream, a);
    if (a.splits > 1) {
        const dim3 grid(static_cast<unsigned>(diff_dkv_join_blocks(bh, a.f.Nk, D, a.splits)));
        if (diff_dkv_slices(a.splits) > 1) hipLaunchKernelGGL((diff_dkv_join_kernel<T, D, 8>), grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL((diff_dkv_join_kernel<T, D, 1>), grid, dim3(kThreads), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_diff_bwd(const DiffBwdArgs& a, int d, bool use_bf16, hipStream_t stream)
{
    if (use_bf16) return d == 32 ? launch_bwd<bf16, 32>(a, stream) : launch_bwd<bf16, 64>(a, stream);
    return d == 32 ? launch_bwd<float, 32>(a, stream) : launch_bwd<float, 64>(a, stream);
}

}  // namespace qta
