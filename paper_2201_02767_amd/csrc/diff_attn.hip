// Differential attention, forward (the mathematics of the tiles is in diff_attn.h).
//
// One pass over the keys with running maxima and sums, S^T = K Q^T so that a lane holds one query's scores and its
// rescaling is a lane's own. The two softmax maps share nothing but V and the rows, so a wave takes one map of 32 NQ
// rows, and the difference is formed once at the end through LDS: a wave that held both maps' results would need twice the
// accumulators and could take only half the rows, reading K and V from LDS twice as often.
#include <atomic>

#include "diff_attn.h"

namespace qta {
namespace {

using namespace diff;

constexpr int kThreads = 256;

// Four waves: wave w takes map w & 1 of the 32 NQ rows of block w >> 1. K_0, K_1 and V come in tiles of BN keys, two in LDS.
template <typename T, int D, int NQ, int BN>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void diff_fwd_kernel(DiffArgs a)
{
    using KT = Tile<T, D>;
    using VT = Tile<T, 2 * D>;
    constexpr int ES = sizeof(T), CT = 2 * D / 32, BM = 64 * NQ;
    constexpr int kK = KT::bytes(BN), kStage = 2 * kK + VT::bytes(BN);
    extern __shared__ __align__(16) unsigned char lds_raw[];
    lds_byte* const lds = (lds_byte*)lds_raw;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int map = wave & 1, rb = wave >> 1, half = lane >> 5;
    const int tiles_n = (a.R + BM - 1) / BM;
    const int logical = xcd_remap(blockIdx.x, gridDim.x);
    const int bh = logical / tiles_n, tile = tiles_n - 1 - (logical - bh * tiles_n);     // the longest rows first
    const int b = bh / a.kv_heads, g = bh - b * a.kv_heads, G = a.heads / a.kv_heads;
    const int row0 = tile * BM, row1 = min(row0 + BM, a.R);
    const DiffRange range = diff_range(a, b);
    const int kend = range.limit(fast_div(row1 - 1, a.div_G)), kmask = range.limit(fast_div(row0, a.div_G));

    // this lane's rows
    int lim[NQ], qi[NQ], qg[NQ];
    Frag<T> qf[NQ][D / 16];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = min(row0 + rb * 32 * NQ + n * 32 + (lane & 31), a.R - 1);
        qi[n] = fast_div(r, a.div_G);
        qg[n] = r - qi[n] * G;
        lim[n] = range.limit(qi[n]);
        const long long at = b * a.qb + qi[n] * a.qn + (2 * (g * G + qg[n]) + map) * a.qh;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[n][s] = global_frag<T>(a.q, at + 16 * s + 8 * half);
    }
    f32x16 acc[NQ][CT];
    float mx[NQ], sum[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        mx[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[n][c] = f32x16{};
    }

    // rows behind the last visible key are read as that key (they are masked)
    auto stage = [&](int k0, lds_byte* at) {
        const int last = kend - 1 - k0;
        const auto kmap0 = tiles::map_resource(byte_at(a.k, b * a.kb + k0 * a.kn + (2 * g) * a.kh, ES));
        const auto kmap1 = tiles::map_resource(byte_at(a.k, b * a.kb + k0 * a.kn + (2 * g + 1) * a.kh, ES));
        const auto vmap = tiles::map_resource(byte_at(a.v, b * a.vb + k0 * a.vn + g * a.vh, ES));
        const uint32_t kstep = static_cast<uint32_t>(a.kn) * ES, vstep = static_cast<uint32_t>(a.vn) * ES;
        auto koff = [&](int r) { return static_cast<uint32_t>(min(r, last)) * kstep; };
        auto voff = [&](int r) { return static_cast<uint32_t>(min(r, last)) * vstep; };
        KT::stage(at, kmap0, BN, wave, 4, lane, koff);
        KT::stage(at + kK, kmap1, BN, wave, 4, lane, koff);
        VT::stage(at + 2 * kK, vmap, BN, wave, 4, lane, voff);
    };

    const uint32_t base0 = lds_address(lds);
    uint32_t krow = KT::row_base(lane), vcol = VT::col_base(lane);
    const int wrow_last = min(row0 + (rb + 1) * 32 * NQ, a.R) - 1;
    const int wend = row0 + rb * 32 * NQ < a.R ? range.limit(fast_div(wrow_last, a.div_G)) : 0;   // this wave's keys
    const int nt = (kend + BN - 1) / BN;
    if (nt > 0) stage(0, lds);
    for (int t = 0; t < nt; ++t) {
        const int k0 = t * BN;
        tiles::wait_lds_loads();
        __syncthreads();
        if (t + 1 < nt) stage(k0 + BN, lds + ((t + 1) & 1) * kStage);
        if (k0 >= wend) continue;
        opaque(krow);
        opaque(vcol);
        const uint32_t kt = base0 + (t & 1) * kStage + map * kK, vt = base0 + (t & 1) * kStage + 2 * kK;
        f32x16 s[BN / 32][NQ];
#pragma unroll
        for (int u = 0; u < BN / 32; ++u) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[u][n] = f32x16{};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                const Frag<T> kf = KT::row_frag(krow, kt, 32 * u, c);
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[u][n] = mma(kf, qf[n][c], s[u][n]);
            }
        }
        if (k0 + BN > kmask) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int u = 0; u < BN / 32; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (k0 + 32 * u + acc_row(r, half) >= lim[n]) s[u][n][r] = -INFINITY;
        }
        Frag<T> p[NQ][BN / 16];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float m = s[0][n][0];
#pragma unroll
            for (int u = 0; u < BN / 32; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) m = fmaxf(m, s[u][n][r]);
            m = fmaxf(mx[n], fmaxf(m, other_half(m)) * a.scale);
            // (a row that has seen nothing yet keeps -inf; its weights are exp2(-inf - 0))
            const float base = m == -INFINITY ? 0.f : m;
            const float alpha = exp2_fast(mx[n] - base);
            mx[n] = m;
            sum[n] *= alpha;
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[n][c] *= alpha;
#pragma unroll
            for (int u = 0; u < BN / 32; ++u) {
                float x[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    x[r] = exp2_fast(fmaf(s[u][n][r], a.scale, -base));
                    sum[n] += x[r];
                }
                p[n][2 * u] = pack_frag<T>(x);
                p[n][2 * u + 1] = pack_frag<T>(x + 8);
            }
        }
#pragma unroll
        for (int w = 0; w < BN / 16; ++w)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const Frag<T> vf = VT::col_frag(vcol, vt, 16 * w, c);
#pragma unroll
                for (int n = 0; n < NQ; ++n) acc[n][c] = mma(vf, p[n][w], acc[n][c]);
            }
    }

    // the second map's normalised result goes to the first map's wave of the same rows, lane by lane
    float* const box = reinterpret_cast<float*>(lds_raw) + rb * (CT * 16 * 64);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float total = sum[n] + other_half(sum[n]);
        const float inv = total > 0.f ? 1.0f / total : 0.f;
        const int r = row0 + rb * 32 * NQ + n * 32 + (lane & 31), h = g * G + qg[n];
        const long long row = (static_cast<long long>(b) * a.Nq + qi[n]) * a.heads + h;
        __syncthreads();
        if (map == 1) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) box[(c * 16 + e) * 64 + lane] = acc[n][c][e] * inv;
        }
        if (r < a.R && a.lse && half == 0)
            a.lse[((static_cast<long long>(b) * a.heads + h) * 2 + map) * a.Nq + qi[n]] =
                total > 0.f ? mx[n] + __builtin_amdgcn_logf(total) : -INFINITY;
        __syncthreads();
        if (map == 0 && r < a.R) {
            const float lam = diff_lambda(a, b, qi[n], h);
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    float o1[4], o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        o1[j] = box[(c * 16 + e + j) * 64 + lane];
                        o[j] = acc[n][c][e + j] * inv - lam * o1[j];
                    }
                    const long long at = row * (2 * D) + 32 * c + acc_row(e, half);
                    store4<T>(a.out, at, o[0], o[1], o[2], o[3]);
                    if (a.out1) store4<T>(a.out1, at, o1[0], o1[1], o1[2], o1[3]);
                }
        }
    }
}

template <typename T, int D, int NQ, int BN>
hipError_t launch_fwd(const DiffArgs& a, hipStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    constexpr int stage = BN * 4 * D * static_cast<int>(sizeof(T));
    constexpr int box = 2 * (2 * D / 32) * 16 * 64 * 4;
    constexpr int lds = 2 * stage > box ? 2 * stage : box;
    const void* fn = reinterpret_cast<const void*>(&diff_fwd_kernel<T, D, NQ, BN>);
    const hipError_t e = set_max_lds_once(fn, configured);
    if (e != hipSuccess) return e;
    const long long blocks = static_cast<long long>((a.R + 64 * NQ - 1) / (64 * NQ)) * a.B * a.kv_heads;
    if (blocks > 0x7FFFFFFFLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL((diff_fwd_kernel<T, D, NQ, BN>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), lds, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_diff_attn(const DiffArgs& a, int d, bool use_bf16, hipStream_t stream)
{
    if (use_bf16) return d == 32 ? launch_fwd<bf16, 32, 1, 64>(a, stream) : launch_fwd<bf16, 64, 1, 64>(a, stream);
    return d == 32 ? launch_fwd<float, 32, 1, 32>(a, stream) : launch_fwd<float, 64, 1, 32>(a, stream);
}

}  // namespace qta
