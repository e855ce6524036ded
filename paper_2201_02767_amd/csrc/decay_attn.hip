// Linear attention with a decay for each head: chunks of tokens through a state (the mathematics is in decay_attn.h).
//
// A workgroup takes one segment of one head's tokens, a wave 32 columns of the state for it, which stay in registers from
// chunk to chunk. Scores come transposed, K Q^T, and the state with its rows in the order of a fragment, so that both are operands
// of the products that make the results, V^T P^T and S^T Q^T, where they lie.
#include <atomic>

#include "decay_attn.h"

namespace qta {
namespace {

using namespace diff;

// x as fragments that sum to it: bf16 two terms of 8 bits each (2^-17 of each value at most is left out) or three (all of it).
template <typename T, int N> struct Terms {
    Frag<T> t[N];
};
template <typename T, int N>
__device__ __forceinline__ Terms<T, N> split_terms(const float* x)
{
    Terms<T, N> r;
    if constexpr (sizeof(T) == 4) {
        r.t[0] = pack_frag<T>(x);
    } else {
        u32x4_t w[N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo = x[2 * i], hi = x[2 * i + 1];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t p = pack2(lo, hi);
                w[n][i] = p;
                if (n + 1 < N) {
                    lo -= tiles::low_half(p);
                    hi -= tiles::high_half(p);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) r.t[n].v = __builtin_bit_cast(bf16x8_t, w[n]);
    }
    return r;
}

__device__ __forceinline__ void unpack_frag(const Frag<float>& f, float* x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = f.v[i];
}
__device__ __forceinline__ void unpack_frag(const Frag<bf16>& f, float* x)
{
    const u32x4_t w = __builtin_bit_cast(u32x4_t, f.v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = tiles::low_half(w[i]);
        x[2 * i + 1] = tiles::high_half(w[i]);
    }
}

// A buffer descriptor of a map from `base` (wave-uniform) on: raw bytes, offsets below 2^31.
__device__ __forceinline__ u32x4_t map_words(const unsigned char* base)
{
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    const int lo = __builtin_amdgcn_readfirstlane(static_cast<int>(p)), hi = __builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32));
    return u32x4_t{static_cast<uint32_t>(lo), static_cast<uint32_t>(hi) & 0xFFFFu, 0x7FFFFFFFu, 0x00020000u};
}

// 16 bytes a lane from the map to LDS, lane i's at byte dst + 16 i. In assembly, which has no register of a lane's to write: of
// the builtin the compiler waits for every load before the next transposed read from LDS, which here are of chunks that landed long before
// (that wait in the middle of a chunk: 200 us for 152 below). wait for them with s_waitcnt vmcnt.
__device__ __forceinline__ void load_lds16_untracked(const u32x4_t& map, uint32_t off, uint32_t dst)
{
    // (nothing else here uses m0; five wait states between a lane operation that wrote the descriptor and the load, one behind m0)
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(map), "s"(dst) : "memory");
}

// log2 of a head's decay, so large at most that products with token counts stay numbers.
__device__ __forceinline__ float decay_log2(const float* log_decay, int h)
{
    const float x = log_decay[h] * 1.44269504088896f;
    return x == x ? fminf(fmaxf(x, -16384.f), 16384.f) : x;
}
__device__ __forceinline__ int decay_length(const int32_t* lens, int b, int N) { return lens ? min(max(lens[b], 0), N) : N; }

// EXACT: what is added to the state keeps 24 bits (bf16: three terms of the weighted values), for a state that the call returns; 16 bits
// (two) do where the state only makes results of 8.
// STATES: only what each segment adds to the state, to a.part. Otherwise the results, from the states before each segment.
template <typename T, int DK, int DV, int C, bool STATES, bool EXACT>
__global__ __launch_bounds__(2 * DV, DK <= 64 ? DECAY_LB : 2) void decay_chunk_kernel(DecayArgs a)
{
    using KT = Tile<T, DK>;
    using VT = Tile<T, DV>;
    constexpr int ES = sizeof(T), W = DV / 32, A = DK / 32, TT = C / 32;
    constexpr int kQ = STATES ? 0 : KT::bytes(C), kK = KT::bytes(C), kStage = kQ + kK + VT::bytes(C);
    constexpr int PT = ES == 2 ? 2 : 1, ST = ES == 2 ? (EXACT ? 3 : 2) : 1;      // terms of scores and states as operands, of what states get
    static_assert(TT <= 2, "the products of one or two tiles of tokens");
    extern __shared__ __align__(1024) unsigned char lds_raw[];
    lds_byte* const lds = (lds_byte*)lds_raw;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, tok = lane & 31;
    // roles, then heads, lie next to each other: they read the same lines
    int x = xcd_remap(blockIdx.x, gridDim.x);
    const int which = x % a.roles;
    x /= a.roles;
    const int y = fast_div(x, a.div_heads), h = x - y * a.heads;
    const int b = fast_div(y, a.div_segs), seg = y - b * a.segs;
    const DecayRole& role = a.role[which];
    const int length = decay_length(a.lens, b, a.N);
    const int t0 = seg * a.seg, t1 = min(t0 + a.seg, length);
    const float g2 = decay_log2(a.log_decay, h);
    const int e1 = role.back ? 0 : 1;                               // 1 - e
    const long long cell = ((static_cast<long long>(b) * a.heads + h) * a.segs + seg) * (DK * DV);

    if constexpr (!STATES) {
        // rows behind the length
        T* const out = static_cast<T*>(role.out);
        for (int n = max(t0, length) + static_cast<int>(threadIdx.x) / (DV / 4); n < min(t0 + a.seg, a.N); n += 8)
            store4<T>(out, ((static_cast<long long>(b) * a.N + n) * a.heads + h) * DV + (threadIdx.x % (DV / 4)) * 4, 0.f, 0.f, 0.f, 0.f);
    }

    // state: register r of tile t holds row 32 t + 16 (r >> 3) + 8 half + (r & 7) of column 32 wave + tok
    f32x16 S[A];
#pragma unroll
    for (int t = 0; t < A; ++t) S[t] = f32x16{};
    auto state_at = [&](int t, int r) {
        return static_cast<long long>(32 * t + 16 * (r >> 3) + 8 * half + (r & 7)) * role.s_row + (32 * wave + tok) * role.s_col;
    };
    if (!STATES && role.state) {
        const float* const from = role.state + cell;
#pragma unroll
        for (int t = 0; t < A; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[t][r] = from[state_at(t, r)];
    }

    // weights: of a score (row acc_row(r) of column tok) on the diagonal tile and on the one before it, of the state in each token,
    // and of rows 16 u + (0 .. 15) of a whole chunk in the state
    float diag[16], before[TT == 2 ? 16 : 1], after = 0.f, come[TT], into[C / 16][8];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int apart = tok - acc_row(r, half);
        diag[r] = apart >= 0 ? exp2f(g2 * apart) * a.scale : 0.f;
        if constexpr (TT == 2) before[r] = exp2f(g2 * (32 - acc_row(r, half)));
    }
    if constexpr (TT == 2) after = exp2f(g2 * tok) * a.scale;
#pragma unroll
    for (int t = 0; t < TT; ++t) come[t] = exp2f(g2 * (32 * t + tok + e1)) * role.f;
    float keep;
    auto weigh = [&](int tokens) {                                  // of a chunk of so many
        keep = exp2f(g2 * tokens);
#pragma unroll
        for (int u = 0; u < C / 16; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 16 * u + 8 * (i >> 2) + 4 * half + (i & 3);
                into[u][i] = j < tokens ? exp2f(g2 * (tokens - j - e1)) * role.u : 0.f;
            }
    };
    weigh(C);

    // Token t of the role's time lies at t, or with time running back at length - 1 - t. Rows behind the last token are read as that.
    // A lane's places within a chunk are the same for all whole ones: only the last chunk, which is staged last, changes them.
    constexpr int RK = 64 / KT::kChunks * W, RV = 64 / VT::kChunks * W, NK = (C + RK - 1) / RK, NV = (C + RV - 1) / RV;   // rows and number of instructions
    uint32_t qoff[STATES ? 1 : NK], koff[NK], voff[NV];
    auto place = [&](int tokens) {
        auto rows = [&](auto& off, int n, int per, int chunks, auto swz, long long stride) {
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const int r = i * per + wave * (64 / chunks) + lane / chunks, m = min(r, tokens - 1);
                off[i] = static_cast<uint32_t>(role.back ? tokens - 1 - m : m) * (static_cast<uint32_t>(stride) * ES) + ((lane % chunks) ^ swz(r)) * 16;
            }
        };
        if constexpr (!STATES) rows(qoff, NK, RK, KT::kChunks, KT::swz, role.qn);
        rows(koff, NK, RK, KT::kChunks, KT::swz, role.kn);
        rows(voff, NV, RV, VT::kChunks, VT::swz, role.vn);
    };
    place(C);
    auto stage = [&](int c0, lds_byte* at) {
        const int tokens = min(C, t1 - c0);
        if (tokens < C) place(tokens);
        const int first = role.back ? length - c0 - tokens : c0;
        auto bring = [&](const auto& off, int n, int per, int chunks, int bytes, const void* x, long long elem, lds_byte* to) {
            const u32x4_t map = map_words(byte_at(x, elem, ES));
            const uint32_t at0 = __builtin_amdgcn_readfirstlane(lds_address(to) + wave * (64 / chunks) * bytes);
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (i * per + wave * (64 / chunks) < C) load_lds16_untracked(map, off[i], at0 + i * per * bytes);
        };
        if constexpr (!STATES) bring(qoff, NK, RK, KT::kChunks, KT::kRow, role.q, b * role.qb + first * role.qn + h * role.qh, at);
        bring(koff, NK, RK, KT::kChunks, KT::kRow, role.k, b * role.kb + first * role.kn + h * role.kh, at + kQ);
        bring(voff, NV, RV, VT::kChunks, VT::kRow, role.v, b * role.vb + first * role.vn + h * role.vh, at + kQ + kK);
    };

    const uint32_t base = lds_address(lds);
    const uint32_t row = base + KT::row_base(lane), kcol = base + kQ + KT::col_base(lane, true), vcol = base + kQ + kK + VT::col_base(lane);
    uint32_t at = 0;
    // D chunks in LDS: one worked on, the others on their way. A wave's loads land in order, so that once no more than those of the
    // D - 2 later chunks are outstanding (kLater: as many as every wave has issued for them at least) the next chunk is there.
    constexpr int D = decay_depth(kStage), kLater = (D - 2) * ((STATES ? 1 : 2) * (C / RK) + C / RV);
    if (t0 < t1) {
        for (int d = 0; d < D - 1 && t0 + d * C < t1; ++d) stage(t0 + d * C, lds + d * kStage);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();
    }
    for (int c0 = t0; c0 < t1; c0 += C) {
        // (what lies there was read before the last barrier)
        const bool more = c0 + (D - 1) * C < t1;
        if (more) stage(c0 + (D - 1) * C, lds + (at == 0 ? (D - 1) * kStage : at - kStage));
        const int left = t1 - c0;
        if (left < C) weigh(left);
        f32x16 o[TT];
        Terms<T, PT> p[3][2];                                       // tiles (0, 0), (1, 0), (1, 1) of the scores
        if constexpr (!STATES) {
            f32x16 s[TT == 2 ? 3 : 1];
#pragma unroll
            for (int t = 0; t < TT; ++t) o[t] = f32x16{};
#pragma unroll
            for (int t = 0; t < (TT == 2 ? 3 : 1); ++t) s[t] = f32x16{};
#pragma unroll
            for (int c = 0; c < DK / 16; ++c) {
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = S[c / 2][8 * (c & 1) + i];
                const Terms<T, PT> st = split_terms<T, PT>(z);
                Frag<T> qf[TT], kf[TT];
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    qf[t] = KT::row_frag(row + at, 0, 32 * t, c);
                    kf[t] = KT::row_frag(row + at, kQ, 32 * t, c);
                }
                s[0] = mma(kf[0], qf[0], s[0]);
                if constexpr (TT == 2) {
                    s[1] = mma(kf[0], qf[1], s[1]);
                    s[2] = mma(kf[1], qf[1], s[2]);
                }
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int n = 0; n < PT; ++n) o[t] = mma(st.t[n], qf[t], o[t]);
            }
#pragma unroll
            for (int t = 0; t < TT; ++t) o[t] *= come[t];
#pragma unroll
            for (int t = 0; t < (TT == 2 ? 3 : 1); ++t)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    float z[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = s[t][8 * w + i] * (TT == 2 && t == 1 ? before[TT == 2 ? 8 * w + i : 0] * after : diag[8 * w + i]);
                    p[t][w] = split_terms<T, PT>(z);
                }
        }
#pragma unroll
        for (int t = 0; t < A; ++t) S[t] *= keep;
#pragma unroll
        for (int u = 0; u < C / 16; ++u) {
            const Frag<T> vf = VT::col_frag(vcol + at, 0, 16 * u, wave);
            if constexpr (!STATES) {
#pragma unroll
                for (int n = 0; n < PT; ++n) {
                    if (u < 2) o[0] = mma(vf, p[0][u & 1].t[n], o[0]);
                    if constexpr (TT == 2) o[1] = mma(vf, p[u < 2 ? 1 : 2][u & 1].t[n], o[1]);
                }
            }
            float z[8];
            unpack_frag(vf, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] *= into[u][i];
            const Terms<T, ST> vt = split_terms<T, ST>(z);
#pragma unroll
            for (int t = 0; t < A; ++t) {
                const Frag<T> kf = KT::col_frag(kcol + at, 0, 16 * u, t);
#pragma unroll
                for (int n = 0; n < ST; ++n) S[t] = mma(kf, vt.t[n], S[t]);
            }
        }
        // the next chunk has landed before this one's results go out, so that nobody waits for these
        if (more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLater) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if constexpr (!STATES) {
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int i = 32 * t + tok;
                if (i < left) {
                    const int n = role.back ? length - 1 - c0 - i : c0 + i;
                    const long long to = ((static_cast<long long>(b) * a.N + n) * a.heads + h) * DV + 32 * wave + 4 * half;
#pragma unroll
                    for (int r = 0; r < 16; r += 4) store4<T>(role.out, to + 2 * r, o[t][r], o[t][r + 1], o[t][r + 2], o[t][r + 3]);
                }
            }
        }
        __syncthreads();
        at = at == (D - 1) * kStage ? 0 : at + kStage;
    }
    float* to = nullptr;
    if constexpr (STATES) to = a.part + static_cast<long long>(which) * a.B * a.heads * a.segs * (DK * DV) + cell;
    else if (role.last) to = role.last + cell;
    if (to) {
#pragma unroll
        for (int t = 0; t < A; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) to[state_at(t, r)] = S[t][r];
    }
}

// The states before each segment, from what each adds: a thread four cells of the state, segment after segment.
__global__ __launch_bounds__(256) void decay_scan_kernel(DecayScanArgs a)
{
    const int quads = a.cells / 4;
    const long long per = static_cast<long long>(a.B) * a.heads * quads;
    const long long item = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (item >= per) return;
    const int role = blockIdx.y;
    const long long bh = item / quads;
    const int quad = static_cast<int>(item - bh * quads);
    const int b = static_cast<int>(bh / a.heads), h = static_cast<int>(bh - static_cast<long long>(b) * a.heads);
    const int length = decay_length(a.lens, b, a.N);
    const float g2 = decay_log2(a.log_decay, h), keep = exp2f(g2 * a.seg);
    f32x4* const part = reinterpret_cast<f32x4*>(a.part) + (role * static_cast<long long>(a.B) * a.heads + bh) * a.segs * quads + quad;
    const float* const state = role ? a.state[1] : a.state[0];
    float* const last = role ? a.last[1] : a.last[0];
    f32x4 S = state ? reinterpret_cast<const f32x4*>(state)[bh * quads + quad] : f32x4{};
    constexpr int kAhead = 8;                                       // segments whose loads are in flight
    for (int s0 = 0; s0 < a.segs; s0 += kAhead) {
        f32x4 add[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) add[i] = part[static_cast<long long>(min(s0 + i, a.segs - 1)) * quads];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = s0 + i;
            if (s >= a.segs) break;
            const int left = length - s * a.seg;
            part[static_cast<long long>(s) * quads] = S;
            if (left > 0) S = S * (left >= a.seg ? keep : exp2f(g2 * left)) + add[i];
        }
    }
    if (last) reinterpret_cast<f32x4*>(last)[bh * quads + quad] = S;
}

// Few tokens: a workgroup holds SV columns of a head's state in registers, a thread four columns of every 1024 / SV-th row, and
// takes token after token. Bound by the states' bytes.
template <typename T, int DK, int DV, int SV>
__global__ __launch_bounds__(256) void decay_step_kernel(DecayStepArgs a)
{
    constexpr int QUADS = SV / 4, GROUPS = 256 / QUADS, ROWS = (DK + GROUPS - 1) / GROUPS;
    static_assert(DK % GROUPS == 0, "every thread has its rows");
    __shared__ float q[kDecayStepTokens][DK], k[kDecayStepTokens][DK], v[kDecayStepTokens][SV];
    __shared__ float part[kDecayStepTokens][4][SV];
    const int slices = DV / SV;
    const int x = blockIdx.x / slices, slice = blockIdx.x - x * slices;
    const int b = fast_div(x, a.div_heads), h = x - b * a.heads;
    const int quad = threadIdx.x % QUADS, group = threadIdx.x / QUADS, length = decay_length(a.lens, b, a.N);
    const long long cell = static_cast<long long>(x) * (DK * DV) + slice * SV + quad * 4;
    f32x4 S[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        S[r] = a.state ? *reinterpret_cast<const f32x4*>(a.state + cell + (group + r * GROUPS) * DV) : f32x4{};
    for (int i = threadIdx.x; i < length * DK; i += 256) {
        const int n = i / DK, c = i - n * DK;
        q[n][c] = Storage<T>::load1(a.q, b * a.qb + n * a.qn + h * a.qh + c) * a.scale;
        k[n][c] = Storage<T>::load1(a.k, b * a.kb + n * a.kn + h * a.kh + c);
    }
    for (int i = threadIdx.x; i < length * SV; i += 256) {
        const int n = i / SV, c = i - n * SV;
        v[n][c] = Storage<T>::load1(a.v, b * a.vb + n * a.vn + h * a.vh + slice * SV + c);
    }
    const float f = exp2f(decay_log2(a.log_decay, h));
    __syncthreads();
    for (int n = 0; n < length; ++n) {
        const f32x4 vn = *reinterpret_cast<const f32x4*>(&v[n][quad * 4]);
        f32x4 o{};
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float kr = k[n][group + r * GROUPS], qr = q[n][group + r * GROUPS];
            S[r] = S[r] * f + vn * kr;
            o += S[r] * qr;
        }
        // the wave's groups of rows lie QUADS lanes apart
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (QUADS <= 8) o[i] += xchg_f32<8>(o[i]);
            if constexpr (QUADS <= 16) o[i] += xchg_f32<16>(o[i]);
            if constexpr (QUADS <= 32) o[i] += xchg_f32<32>(o[i]);
        }
        if ((threadIdx.x & 63) < QUADS) *reinterpret_cast<f32x4*>(&part[n][threadIdx.x >> 6][quad * 4]) = o;
    }
    if (a.last) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) *reinterpret_cast<f32x4*>(a.last + cell + (group + r * GROUPS) * DV) = S[r];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.N * SV; i += 256) {
        const int n = i / SV, c = i - n * SV;
        const float o = n < length ? (part[n][0][c] + part[n][1][c]) + (part[n][2][c] + part[n][3][c]) : 0.f;
        Storage<T>::store1(a.out, ((static_cast<long long>(b) * a.N + n) * a.heads + h) * DV + slice * SV + c, o);
    }
}

template <typename T, int DK, int DV, bool STATES, bool EXACT>
hipError_t launch_exact(const DecayArgs& a, hipStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    constexpr int C = decay_chunk(sizeof(T) == 2), stage = C * ((STATES ? 1 : 2) * DK + DV) * static_cast<int>(sizeof(T)), lds = decay_depth(stage) * stage;
    const auto kernel = &decay_chunk_kernel<T, DK, DV, C, STATES, EXACT>;
    const hipError_t e = set_max_lds_once(reinterpret_cast<const void*>(kernel), configured);
    if (e != hipSuccess) return e;
    DecayArgs p = a;
    p.div_segs = make_fastdiv(a.segs);
    p.div_heads = make_fastdiv(a.heads);
    const long long blocks = static_cast<long long>(a.roles) * a.B * a.heads * a.segs;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(2 * DV), lds, stream, p);
    return hipGetLastError();
}

template <typename T, int DK, int DV, bool STATES>
hipError_t launch(const DecayArgs& a, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        if (!a.exact) return launch_exact<T, DK, DV, STATES, false>(a, stream);
    }
    return launch_exact<T, DK, DV, STATES, true>(a, stream);
}

template <typename T, int DK, int DV>
hipError_t launch_step(const DecayStepArgs& a, hipStream_t stream)
{
    DecayStepArgs p = a;
    p.div_heads = make_fastdiv(a.heads);
    constexpr int SV = DV < 64 ? DV : 64;
    const long long blocks = static_cast<long long>(a.B) * a.heads * (DV / SV);
    hipLaunchKernelGGL((decay_step_kernel<T, DK, DV, SV>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

// f.template operator()<T, DK, DV>() for the call's type and sizes
template <typename T, int DK, typename F>
hipError_t by_dv(int dv, F f)
{
    return dv == 32 ? f.template run<T, DK, 32>() : dv == 64 ? f.template run<T, DK, 64>() : f.template run<T, DK, 128>();
}
template <typename T, typename F>
hipError_t by_dk(int dk, int dv, F f)
{
    return dk == 32 ? by_dv<T, 32>(dv, f) : dk == 64 ? by_dv<T, 64>(dv, f) : by_dv<T, 128>(dv, f);
}
template <typename F>
hipError_t by_type(int dk, int dv, bool use_bf16, F f)
{
    return use_bf16 ? by_dk<bf16>(dk, dv, f) : by_dk<float>(dk, dv, f);
}

struct StepLauncher {
    const DecayStepArgs& a;
    hipStream_t stream;
    template <typename T, int DK, int DV> hipError_t run() const { return launch_step<T, DK, DV>(a, stream); }
};
template <bool STATES>
struct ChunkLauncher {
    const DecayArgs& a;
    hipStream_t stream;
    template <typename T, int DK, int DV> hipError_t run() const { return launch<T, DK, DV, STATES>(a, stream); }
};

}  // namespace

hipError_t launch_decay_step(const DecayStepArgs& a, int dk, int dv, bool use_bf16, hipStream_t stream)
{
    return by_type(dk, dv, use_bf16, StepLauncher{a, stream});
}

hipError_t launch_decay_states(const DecayArgs& a, int dk, int dv, bool use_bf16, hipStream_t stream)
{
    return by_type(dk, dv, use_bf16, ChunkLauncher<true>{a, stream});
}

hipError_t launch_decay_chunks(const DecayArgs& a, int dk, int dv, bool use_bf16, hipStream_t stream)
{
    return by_type(dk, dv, use_bf16, ChunkLauncher<false>{a, stream});
}

hipError_t launch_decay_scan(const DecayScanArgs& a, int roles, hipStream_t stream)
{
    const long long items = static_cast<long long>(a.B) * a.heads * (a.cells / 4);
    hipLaunchKernelGGL(decay_scan_kernel, dim3(static_cast<unsigned>((items + 255) / 256), static_cast<unsigned>(roles)), dim3(256), 0,
                       stream, a);
    return hipGetLastError();
}

}  // namespace qta
