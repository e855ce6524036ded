// Differential attention, forward (the mathematics of the tiles is in diff_attn.h).
//
// One pass over the keys with running maxima and sums, S^T = K Q^T so that a lane holds one query's scores and its
// rescaling is a lane's own. The two softmax maps share nothing but V and the rows, so a wave takes one map of 32 rows, and
// the difference is formed once at the end through LDS.
//
// What bounds it: long prompts the matrix and the vector units together, at the clock that their power leaves (2 x 8192 causal
// tokens, 16 heads over 4, d = 64, bf16: 792 to 819 us, 1007 to 1041 TFLOP/s of products at 1.9 GHz, where a large library
// product reaches 1305); single tokens the caches' bytes (1.6 GB: 270 us, 6 TB/s). Tried beside 830 us for prompts on one
// card: four waves a SIMD with a few spills 806 us, but 264 instead of 236 for the forward of training, which writes more; one
// wave over 64 rows 793 us, none gained in training; tiles of 64 keys 895 us; a pipeline over three tiles that alternates
// matrix and vector instructions 930 us.
#include <atomic>
#include <type_traits>

#include "diff_attn.h"

namespace qta {
namespace {

using namespace diff;

constexpr int kThreads = kDiffThreads;

// Maxima lag: a row's running maximum is raised only when a tile exceeds it by 2^8 or more, so that most tiles rescale
// nothing. Weights then go up to 2^8, which costs neither fp32 sums nor bf16 weights any of their bits.
constexpr float kLag = 8.0f;

// Four waves over a tile of 64 rows: wave w takes map w & 1 of the 32 rows of block w >> 1. With KEYS, for calls of few
// rows, over a tile of 32 rows: w >> 1 is then the half of every key tile that the wave takes. K_0, K_1 and V come in tiles of BN
// keys, two of them in LDS. With a.splits > 1 a workgroup takes one part of its rows' keys and leaves the results as they
// are, with their maxima and sums, to diff_join_kernel.
template <typename T, int D, int BN, bool KEYS>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? (KEYS ? 2 : 3) : 1) void diff_fwd_kernel(DiffArgs a)
{
    using KT = Tile<T, D>;
    using VT = Tile<T, 2 * D>;
    constexpr int ES = sizeof(T), CT = 2 * D / 32, BM = KEYS ? 32 : 64, U = KEYS ? BN / 64 : BN / 32;   // 32-key blocks of a wave
    constexpr int kK = KT::bytes(BN), kStage = 2 * kK + VT::bytes(BN);
    static_assert(U >= 1, "a block of keys for every wave");
    // bf16 terms of a weight. One is off by 2^-9, as the result's rounding is, and more where the two maps cancel: 0.0024 to
    // 0.0026 from the exact result for 0.0017 by rounding alone. Few rows wait for their keys' bytes, and take two (16 bits,
    // 0.0017; the long caches 276 us for 273); for prompts four units of product more for 12 would buy it.
    constexpr int TERMS = KEYS && ES == 2 ? 2 : 1;
    extern __shared__ __align__(1024) unsigned char lds_raw[];
    lds_byte* const lds = (lds_byte*)lds_raw;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int map = wave & 1, rb = KEYS ? 0 : wave >> 1, kb = KEYS ? wave >> 1 : 0, half = lane >> 5;
    const int tiles_n = (a.R + BM - 1) / BM;
    const int logical = xcd_remap(blockIdx.x, gridDim.x);
    const int work = logical / a.splits, split = logical - work * a.splits;
    const int bh = work / tiles_n, tile = tiles_n - 1 - (work - bh * tiles_n);     // the longest rows first
    const int b = bh / a.kv_heads, g = bh - b * a.kv_heads, G = a.heads / a.kv_heads;
    const int row0 = tile * BM, row1 = min(row0 + BM, a.R);
    const DiffRange range = diff_range(a, b);
    const int kend = range.limit(fast_div(row1 - 1, a.div_G)), kmask = range.limit(fast_div(row0, a.div_G));

    // this lane's row
    const int rr = row0 + rb * 32 + (lane & 31), r = min(rr, a.R - 1);
    const int qi = fast_div(r, a.div_G), h = g * G + r - qi * G, lim = range.limit(qi);
    Frag<T> qf[D / 16];
    const long long qat = range.read_as(qi, a.Nq);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = global_frag<T>(a.q, b * a.qb + qat * a.qn + (2 * h + map) * a.qh + 16 * s + 8 * half);
    f32x16 acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = f32x16{};
    float mx = -INFINITY, sum = 0.f;

    // rows behind the last visible key are read as that key (they are masked)
    auto stage = [&](int k0, lds_byte* at) {
        const int last = kend - 1 - k0;
        const auto kmap0 = tiles::map_resource(byte_at(a.k, b * a.kb + k0 * a.kn + (2 * g) * a.kh, ES));
        const auto kmap1 = tiles::map_resource(byte_at(a.k, b * a.kb + k0 * a.kn + (2 * g + 1) * a.kh, ES));
        const auto vmap = tiles::map_resource(byte_at(a.v, b * a.vb + k0 * a.vn + g * a.vh, ES));
        const uint32_t kstep = static_cast<uint32_t>(a.kn) * ES, vstep = static_cast<uint32_t>(a.vn) * ES;
        auto koff = [&](int x) { return static_cast<uint32_t>(min(x, last)) * kstep; };
        auto voff = [&](int x) { return static_cast<uint32_t>(min(x, last)) * vstep; };
        KT::stage(at, kmap0, BN, wave, 4, lane, koff);
        KT::stage(at + kK, kmap1, BN, wave, 4, lane, koff);
        VT::stage(at + 2 * kK, vmap, BN, wave, 4, lane, voff);
    };

    // this wave's keys, and this workgroup's part of the tiles
    const int wend = row0 + rb * 32 < a.R ? range.limit(fast_div(min(row0 + rb * 32 + 32, a.R) - 1, a.div_G)) : 0;
    const int all = (kend + BN - 1) / BN;
    const int t0 = static_cast<int>(static_cast<long long>(all) * split / a.splits);
    const int t1 = static_cast<int>(static_cast<long long>(all) * (split + 1) / a.splits);
    // (whole rows are added, so that the bases keep their bits below)
    const uint32_t krow = lds_address(lds) + KT::row_base(lane) + map * kK + kb * (BN / 2) * KT::kRow,
                   vcol = lds_address(lds) + VT::col_base(lane) + 2 * kK + kb * (BN / 2) * VT::kRow;
    auto keys = [&](int k0, auto odd) {
        constexpr uint32_t at = odd.value * kStage;
        f32x16 s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = f32x16{};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) s[u] = mma(KT::row_frag(krow, at, 32 * u, c), qf[c], s[u]);
        }
        if (k0 + BN > kmask) {
            branch_here();
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k0 + kb * (BN / 2) + 32 * u + acc_row(e, half) >= lim) s[u][e] = -INFINITY;
        }
        float m = s[0][0];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) m = fmaxf(m, s[u][e]);
        m = fmaxf(m, other_half(m)) * a.scale;
        if (__any(m > mx + kLag)) {
            m = fmaxf(m, mx);
            const float alpha = exp2_fast(mx - (m == -INFINITY ? 0.f : m));
            mx = m;
            sum *= alpha;
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[c] *= alpha;
        }
        // (a row that has seen nothing yet keeps -inf: its weights are exp2(-inf - 0))
        const float base = mx == -INFINITY ? 0.f : -mx;
        Frag<T> p[2 * U], rest[2 * U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[e] = exp2_fast(fmaf(s[u][e], a.scale, base));
                sum += x[e];
            }
            p[2 * u] = pack_frag<T>(x);
            p[2 * u + 1] = pack_frag<T>(x + 8);
            if constexpr (TERMS == 2) {
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] -= static_cast<float>(p[2 * u + e / 8].v[e % 8]);
                rest[2 * u] = pack_frag<T>(x);
                rest[2 * u + 1] = pack_frag<T>(x + 8);
            }
        }
#pragma unroll
        for (int w = 0; w < 2 * U; ++w)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const Frag<T> x = VT::col_frag(vcol, at, 16 * w, c);
                acc[c] = mma(x, p[w], acc[c]);
                if constexpr (TERMS == 2) acc[c] = mma(x, rest[w], acc[c]);
            }
    };
    if (t0 < t1) stage(t0 * BN, lds);
    for (int t = t0; t < t1; t += 2) {
        tiles::wait_lds_loads();
        __syncthreads();
        if (t + 1 < t1) stage((t + 1) * BN, lds + kStage);
        if (t * BN < wend) keys(t * BN, std::integral_constant<int, 0>{});
        if (t + 1 >= t1) break;
        tiles::wait_lds_loads();
        __syncthreads();
        if (t + 2 < t1) stage((t + 2) * BN, lds);
        if ((t + 1) * BN < wend) keys((t + 1) * BN, std::integral_constant<int, 1>{});
    }
    sum += other_half(sum);

    // results pass between waves of the same rows through LDS, lane by lane
    constexpr int kBox = (CT * 16 + 2) * 64;
    float* const boxes = reinterpret_cast<float*>(lds_raw);
    if constexpr (KEYS) {
        float* const box = boxes + map * kBox + lane;
        __syncthreads();
        if (kb == 1) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) box[(c * 16 + e) * 64] = acc[c][e];
            box[CT * 16 * 64] = mx;
            box[(CT * 16 + 1) * 64] = sum;
        }
        __syncthreads();
        if (kb == 0) {
            const float m1 = box[CT * 16 * 64], m = fmaxf(mx, m1), base = m == -INFINITY ? 0.f : m;
            const float f0 = exp2_fast(mx - base), f1 = exp2_fast(m1 - base);
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[c][e] = acc[c][e] * f0 + box[(c * 16 + e) * 64] * f1;
            sum = sum * f0 + box[(CT * 16 + 1) * 64] * f1;
            mx = m;
        }
    }
    if (a.splits > 1) {
        if (kb == 1 || rr >= a.R) return;
        const long long at = (((static_cast<long long>(split) * a.B * a.kv_heads + bh) * 2 + map) * a.R + r);
        if (half == 0) *reinterpret_cast<float2*>(a.part_sums + at * 2) = make_float2(mx, sum);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                store4<float>(a.part, at * (2 * D) + 32 * c + acc_row(e, half), acc[c][e], acc[c][e + 1], acc[c][e + 2], acc[c][e + 3]);
        return;
    }
    const float inv = sum > 0.f ? 1.0f / sum : 0.f;
    const long long row = (static_cast<long long>(b) * a.Nq + qi) * a.heads + h;
    float* const box = boxes + rb * kBox + lane;
    __syncthreads();
    if (map == 1 && kb == 0) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) box[(c * 16 + e) * 64] = acc[c][e] * inv;
    }
    if (rr < a.R && a.lse && half == 0 && kb == 0)
        a.lse[((static_cast<long long>(b) * a.heads + h) * 2 + map) * a.Nq + qi] =
            sum > 0.f ? mx + __builtin_amdgcn_logf(sum) : -INFINITY;
    __syncthreads();
    if (map == 1 || kb == 1 || rr >= a.R) return;
    const float lam = sum > 0.f ? diff_lambda(a, b, qi, h) : 0.f;      // (a row without a key: whatever its weight is)
    T* const out = static_cast<T*>(a.out) + row * (2 * D) + 4 * half;
    float* const maps = a.maps + row * (4 * D) + 4 * half;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            float o0[4], o1[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                o0[j] = acc[c][e + j] * inv;
                o1[j] = box[(c * 16 + e + j) * 64];
            }
            const int ch = 32 * c + 2 * e;
            store4<T>(out, ch, o0[0] - lam * o1[0], o0[1] - lam * o1[1], o0[2] - lam * o1[2], o0[3] - lam * o1[3]);
            if (a.maps) {
                store4<float>(maps, ch, o0[0], o0[1], o0[2], o0[3]);
                store4<float>(maps, 2 * D + ch, o1[0], o1[1], o1[2], o1[3]);
            }
        }
}

// The parts' results joined: a wave a row, lane s holding the maxima and sums of part s (at most 64), every lane D / 32
// channels of both maps.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_join_kernel(DiffArgs a)
{
    constexpr int V = D / 32;
    typedef float piece __attribute__((ext_vector_type(V)));
    const int lane = threadIdx.x & 63;
    const long long rows = static_cast<long long>(a.B) * a.kv_heads * a.R;
    const long long item = static_cast<long long>(blockIdx.x) * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= rows) return;
    const int bh = static_cast<int>(item / a.R);
    const int r = static_cast<int>(item - static_cast<long long>(bh) * a.R), G = a.heads / a.kv_heads;
    const int b = bh / a.kv_heads, qi = fast_div(r, a.div_G), h = (bh - b * a.kv_heads) * G + r - qi * G;
    const long long step = 2 * rows;
    float f[2], inv[2], top[2], sum[2];
    const float* x[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const long long at = (static_cast<long long>(bh) * 2 + m) * a.R + r;
        const float2 ms = lane < a.splits ? reinterpret_cast<const float2*>(a.part_sums)[at + lane * step] : make_float2(-INFINITY, 0.f);
        top[m] = wave_max_fast(ms.x);
        f[m] = exp2_fast(ms.x - (top[m] == -INFINITY ? 0.f : top[m]));
        sum[m] = wave_sum_fast(ms.y * f[m]);
        inv[m] = sum[m] > 0.f ? 1.0f / sum[m] : 0.f;
        x[m] = a.part + at * (2 * D) + lane * V;
    }
    piece o[2] = {};
    // four parts' loads in flight together (behind the last part: that one again, with the weight 0 of its lane)
    for (int s = 0; s < a.splits; s += 4) {
        piece y[4][2];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int m = 0; m < 2; ++m)
                y[j][m] = *reinterpret_cast<const piece*>(x[m] + min(s + j, a.splits - 1) * step * (2 * D));
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int m = 0; m < 2; ++m) o[m] += y[j][m] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f[m]), s + j));
    }
    const float lam = sum[1] > 0.f ? diff_lambda(a, b, qi, h) : 0.f;
    const long long row = (static_cast<long long>(b) * a.Nq + qi) * a.heads + h;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float o0 = o[0][v] * inv[0], o1 = o[1][v] * inv[1];
        Storage<T>::store1(a.out, row * (2 * D) + lane * V + v, o0 - lam * o1);
        if (a.maps) {
            a.maps[row * (4 * D) + lane * V + v] = o0;
            a.maps[row * (4 * D) + 2 * D + lane * V + v] = o1;
        }
    }
    if (a.lse && lane < 2) {
        const float t = lane ? top[1] : top[0], z = lane ? sum[1] : sum[0];
        a.lse[((static_cast<long long>(b) * a.heads + h) * 2 + lane) * a.Nq + qi] = z > 0.f ? t + __builtin_amdgcn_logf(z) : -INFINITY;
    }
}

template <typename T, int D, int BN, bool KEYS>
hipError_t launch_fwd(const DiffArgs& a, hipStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    constexpr int stage = BN * 4 * D * static_cast<int>(sizeof(T));
    constexpr int boxes = 2 * (2 * D / 32 * 16 + 2) * 64 * 4;
    constexpr int lds = 2 * stage > boxes ? 2 * stage : boxes;
    const void* fn = reinterpret_cast<const void*>(&diff_fwd_kernel<T, D, BN, KEYS>);
    const hipError_t e = set_max_lds_once(fn, configured);
    if (e != hipSuccess) return e;
    const long long groups = static_cast<long long>(a.B) * a.kv_heads;
    const dim3 grid(static_cast<unsigned>(diff_fwd_blocks(groups, a.R, {KEYS, a.splits})));
    hipLaunchKernelGGL((diff_fwd_kernel<T, D, BN, KEYS>), grid, dim3(kThreads), lds, stream, a);
    if (a.splits > 1)
        hipLaunchKernelGGL((diff_join_kernel<T, D>), dim3(static_cast<unsigned>(diff_join_blocks(groups, a.R))), dim3(kThreads), 0,
                           stream, a);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_type(const DiffArgs& a, hipStream_t stream)
{
    if (a.keys_apart) return launch_fwd<T, D, 64, true>(a, stream);
    // tiles of 64 keys where they leave LDS for four workgroups a unit: 33 us against 38 for 3 x 1031 bf16 tokens over 1777
    return launch_fwd<T, D, sizeof(T) == 2 && D == 32 ? 64 : 32, false>(a, stream);
}

}  // namespace

hipError_t launch_diff_attn(const DiffArgs& a, int d, bool use_bf16, hipStream_t stream)
{
    if (use_bf16) return d == 32 ? launch_type<bf16, 32>(a, stream) : launch_type<bf16, 64>(a, stream);
    return d == 32 ? launch_type<float, 32>(a, stream) : launch_type<float, 64>(a, stream);
}

}  // namespace qta
