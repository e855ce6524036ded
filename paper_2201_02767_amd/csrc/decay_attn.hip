// Linear attention with a decay for each head: chunks of tokens through a state (the mathematics is in decay_attn.h).
//
// A workgroup takes one segment of one head's tokens, a wave 32 columns of the state for it, which stay in registers from
// chunk to chunk. Scores come transposed, K Q^T, and the state with its rows in the order of a fragment, so that both are operands
// of the products that make the results, V^T P^T and S^T Q^T, where they lie.
//
// What bounds them. 65536 tokens, 16 heads of 64/128, bf16: states 89 to 104 us (403 MB, 3.9 to 4.5 TB/s), results 185 to 231 (820 MB; without
// any product 197, without stores 120), both at the clock that their power leaves, which a run of passes lowers. 2 x 8192 tokens, 16 heads of
// 128, bf16, backward: results 195 to 226 us, vector units at work in 56% of the cycles and matrix units in 41%: what is split into terms.
// Few or short sequences wait for a chunk's chain of products, 0.5 us in bf16 and 1.1 in fp32 with 32 channels, and for three launches.
// Tried, with two terms in what states get: a state brought to the present every eight chunks instead of every one (a branch in the chunk:
// 233 us for 214), results through LDS for whole lines (registers go to memory at 128 x 128: 239), stores past the caches (240 for 220 of the
// prompts).
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
// (that wait in the middle of a chunk: 130 us for 105 of the states of 65536 tokens). Wait for them with s_waitcnt vmcnt.
__device__ __forceinline__ void load_lds16_untracked(const u32x4_t& map, uint32_t off, uint32_t dst)
{
    // (five wait states between a lane operation that wrote the descriptor and the load, one behind m0. The compiler takes no m0 on a list of what
    // is overwritten, so it is put back)
    uint32_t kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_nop 3\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "v"(off), "s"(map), "s"(dst) : "memory");
}

// log2 of a head's decay, so large at most that products with token counts stay numbers.
__device__ __forceinline__ float decay_log2(const float* log_decay, int h)
{
    const float x = log_decay[h] * 1.44269504088896f;
    return x == x ? fminf(fmaxf(x, -16384.f), 16384.f) : x;
}
__device__ __forceinline__ int decay_length(const int32_t* lens, int b, int N) { return lens ? min(max(lens[b], 0), N) : N; }

// Column tok of a result, 32 rows, as 32 neighbours from element `at` on. bf16: a lane takes 16 of them, by exchanging what lies between
// with the other half's.
template <typename T>
__device__ __forceinline__ void store_tile(void* base, long long at, const f32x16& o)
{
    const int half = (threadIdx.x >> 5) & 1;
    if constexpr (sizeof(T) == 2) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2(o[2 * i], o[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto x = __builtin_amdgcn_permlane32_swap(w[i], w[i + 4], false, false);
            w[i] = x[0];
            w[i + 4] = x[1];
        }
        u32x4_t* const to = reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(base) + at + 16 * half);
        to[0] = u32x4_t{w[0], w[1], w[4], w[5]};
        to[1] = u32x4_t{w[2], w[3], w[6], w[7]};
    } else {
#pragma unroll
        for (int r = 0; r < 16; r += 4) store4<float>(base, at + 2 * r + 4 * half, o[r], o[r + 1], o[r + 2], o[r + 3]);
    }
}

// What is added to the state keeps 24 bits (bf16: three terms of the weighted values), whether or not the call returns it: results are the
// same bits either way. (With two where the state only makes results: 1.08e-4 of them, as a norm, off the rounded exact ones at 2 x 8192
// tokens, 16 heads of 128; with three 0.94e-4, of which the scores' and states' own two terms make the rest. A step takes 355 and 387 us.)
// STATES: only what each segment adds to the state, to a.part. Otherwise the results, from the states before each segment.
template <typename T, int DK, int DV, bool STATES>
__global__ __launch_bounds__(2 * DV, decay_waves(sizeof(T) == 2, DK, DV)) void decay_chunk_kernel(DecayArgs a)
{
    using KT = Tile<T, DK>;
    using VT = Tile<T, DV>;
    constexpr int ES = sizeof(T), W = DV / 32, A = DK / 32, C = kDecayChunk;
    constexpr int kQ = STATES ? 0 : KT::bytes(C), kK = KT::bytes(C), kStage = kQ + kK + VT::bytes(C);
    constexpr int PT = ES == 2 ? 2 : 1, ST = ES == 2 ? 3 : 1;      // terms of scores and states as operands, of what states get
    constexpr int D = decay_depth(kStage);
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

    // Weights, in LDS behind the chunks (registers are what keeps waves off the units): of a score on the diagonal tile (row acc_row(r) of
    // column tok), of token j in the state of a whole chunk and of the last one, which may be shorter; in registers: of the state in each token
    const int tail = t1 > t0 ? (t1 - t0 - 1) % C + 1 : C;
    lds_byte* const tables = lds + D * kStage;
    for (int x = threadIdx.x; x < 64 * 16; x += 2 * DV) {           // [r / 4][lane][r % 4]
        const int l = (x >> 2) & 63, r = (x >> 8) * 4 + (x & 3), apart = (l & 31) - acc_row(r, l >> 5);
        *(lds_ptr<float>)(tables + x * 4) = apart >= 0 ? exp2f(g2 * apart) * a.scale : 0.f;
    }
    for (int x = threadIdx.x; x < 2 * C; x += 2 * DV) {             // [whole, last][16 u + 8 (lane / 32) + i], in the order of a column fragment
        const int y = x & (C - 1), j = (y & ~15) + 8 * ((y >> 2) & 1) + 4 * ((y >> 3) & 1) + (y & 3), n = x < C ? C : tail;
        *(lds_ptr<float>)(tables + 4096 + x * 4) = j < n ? exp2f(g2 * (n - j - e1)) * role.u : 0.f;
    }
    const float come = exp2f(g2 * (tok + e1)) * role.f, keep_whole = exp2f(g2 * C), keep_last = exp2f(g2 * tail);

    // Token t of the role's time lies at t, or with time running back at length - 1 - t. Rows behind the last token are read as that.
    // A lane's places within a chunk are the same for all whole ones.
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
    int placed = 0;
    auto stage = [&](int c0, lds_byte* at) {
        const int tokens = min(C, t1 - c0);
        if (tokens != placed) place(placed = tokens);
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
    constexpr int kLater = (D - 2) * ((STATES ? 1 : 2) * (C / RK) + C / RV);
    // The results' chunks come in the order of time. What a segment adds to the state is summed from its last chunk to its first, with
    // weights that go to the segment's end: then the results' launch, which starts at the segments' first chunks, finds those in the
    // memory's cache, where they were read last.
    const int chunks = t0 < t1 ? (t1 - t0 + C - 1) / C : 0;
    auto start = [&](int x) { return t0 + (STATES ? chunks - 1 - x : x) * C; };
    if (chunks > 0) {
        for (int d = 0; d < D - 1 && d < chunks; ++d) stage(start(d), lds + d * kStage);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();
    }
    for (int x = 0; x < chunks; ++x) {
        // (what lies there was read before the last barrier)
        const int c0 = start(x);
        const bool more = x + D - 1 < chunks;
        if (more) stage(start(x + D - 1), lds + (at == 0 ? (D - 1) * kStage : at - kStage));
        const int left = t1 - c0;
        f32x16 o{};
        Terms<T, PT> p[2];
        if constexpr (!STATES) {
            f32x16 s{};
#pragma unroll
            for (int c = 0; c < DK / 16; ++c) {
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = S[c / 2][8 * (c & 1) + i];
                const Terms<T, PT> st = split_terms<T, PT>(z);
                const Frag<T> qf = KT::row_frag(row + at, 0, 0, c);
                s = mma(KT::row_frag(row + at, kQ, 0, c), qf, s);
#pragma unroll
                for (int n = 0; n < PT; ++n) o = mma(st.t[n], qf, o);
            }
            o *= come;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const f32x4 d = *(lds_ptr<f32x4>)(tables + (8 * w + i) / 4 * 1024 + lane * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[i + e] = s[8 * w + i + e] * d[e];
                }
                p[w] = split_terms<T, PT>(z);
            }
        }
        const float keep = left >= C ? keep_whole : keep_last;
        lds_byte* const into = tables + 4096 + (left >= C ? 0 : 4 * C) + half * 32;
        const float far = STATES ? exp2f(g2 * max(left - C, 0)) : 1.f;
        if constexpr (!STATES) {
#pragma unroll
            for (int t = 0; t < A; ++t) S[t] *= keep;
        }
#pragma unroll
        for (int u = 0; u < C / 16; ++u) {
            const Frag<T> vf = VT::col_frag(vcol + at, 0, 16 * u, wave);
            if constexpr (!STATES) {
#pragma unroll
                for (int n = 0; n < PT; ++n) o = mma(vf, p[u].t[n], o);
            }
            float z[8];
            unpack_frag(vf, z);
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const f32x4 w = *(lds_ptr<f32x4>)(into + u * 64 + i * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[i + e] *= STATES ? w[e] * far : w[e];
            }
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
            if (tok < left) {
                const int n = role.back ? length - 1 - c0 - tok : c0 + tok;
                store_tile<T>(role.out, ((static_cast<long long>(b) * a.N + n) * a.heads + h) * DV + 32 * wave, o);
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

// The states before each segment, from what each adds: a thread four cells of the state, segment after segment. Bound by the latency of
// its loads (32 segments of 16 states of 64 x 128: 9 to 10 us, of 32 of 128 x 128 11; sixteen segments' loads at once, in branches, 32).
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
    // the next four segments' loads are in flight while four are added
    constexpr int kAhead = 4;
    f32x4 add[kAhead], next[kAhead];
    auto fetch = [&](f32x4 (&x)[kAhead], int s0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = part[static_cast<long long>(min(s0 + i, a.segs - 1)) * quads];
    };
    fetch(add, 0);
    for (int s0 = 0; s0 < a.segs; s0 += kAhead) {
        fetch(next, s0 + kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int left = length - (s0 + i) * a.seg;
            if (s0 + i < a.segs) part[static_cast<long long>(s0 + i) * quads] = S;
            if (left >= a.seg) S = S * keep + add[i];
            else if (left > 0) S = S * exp2f(g2 * left) + add[i];
            add[i] = next[i];
        }
    }
    if (last) reinterpret_cast<f32x4*>(last)[bh * quads + quad] = S;
}

// Few tokens: a workgroup holds SV columns of a head's state in registers, a thread four columns of every 1024 / SV-th row, and
// takes token after token. Bound by the states' bytes (64 x 32 heads of 128 x 128, one token: 44 us, 6.1 TB/s), and in small calls by the
// launch (3.8 us).
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

template <typename T, int DK, int DV, bool STATES>
hipError_t launch(const DecayArgs& a, hipStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    constexpr int stage = kDecayChunk * ((STATES ? 1 : 2) * DK + DV) * static_cast<int>(sizeof(T)), lds = decay_depth(stage) * stage + kDecayTables;
    const auto kernel = &decay_chunk_kernel<T, DK, DV, STATES>;
    const hipError_t e = set_max_lds_once(reinterpret_cast<const void*>(kernel), configured);
    if (e != hipSuccess) return e;
    DecayArgs p = a;
    p.div_segs = make_fastdiv(a.segs);
    p.div_heads = make_fastdiv(a.heads);
    const long long blocks = static_cast<long long>(a.roles) * a.B * a.heads * a.segs;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(2 * DV), lds, stream, p);
    return hipGetLastError();
}

template <typename T, int DK, int DV>
hipError_t launch_step(const DecayStepArgs& a, hipStream_t stream)
{
    DecayStepArgs p = a;
    p.div_heads = make_fastdiv(a.heads);
    constexpr int SV = DV < 64 ? DV : 64;
    static_assert(DV / SV == decay_step_slices(DV), "as the launches are checked");
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
