// Rotary positions: pairs of channels turned by an angle that is linear in the token's position.
//
//   y1 = m (x1 cos t - x2 sin t),   y2 = m (x2 cos t + x1 sin t),   t = position * freqs[pair]
//
// The gradient is the turn by -t. Bound by memory: every element is read and written once, so a workgroup takes
// whole tokens, makes each (token, pair) cosine and sine once into LDS for all heads of both tensors, and then streams the
// heads in 16-byte pieces (2 x 16384 tokens, 32 + 8 heads of 128, 64 turned, bf16: 5.1 TB/s, as a large copy; one thread's two
// items at a time; one 136 us, four 160). Angles are products in 64 bits of which only the fraction of a turn is kept: at position
// 10^6 an fp32 product would be off by 0.06 radians, this one by 10^-9, and by the rounding of that fraction to fp32, 10^-7 at most
// (fp32 results: 3.8e-8 off, with cosines rounded from fp64 3.0e-8). The turn itself is in fp32, rounded once.
#include <algorithm>

#include "diff_attn.h"

namespace qta {
namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 2;      // items of a thread whose loads are in flight together

// Position of a token on an axis.
__device__ __forceinline__ int token_position(const RotaryArgs& a, int token, int axis)
{
    const int b = fast_div(token, a.div_N), n = token - b * a.N;
    if (a.pos) return a.pos[b * a.pos_b + static_cast<long long>(n) * a.axes + axis];
    if (a.axes == 1) return a.start + n;
    const int y = fast_div(n, a.div_W);
    return axis == 0 ? y : n - y * a.width;
}

// V elements at element e of `base`, and back. What is written is read by a later kernel only: stores that ask for no place
// in the caches take 132 us for 671 MB in and out, ordinary ones 140.
template <typename T, int V>
struct Piece {
    float x[V];
    __device__ __forceinline__ void load(const void* base, long long e)
    {
        if constexpr (V * sizeof(T) == 16) {
            Storage<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(base) + e), x);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = Storage<T>::load1(base, e + i);
        }
    }
    __device__ __forceinline__ void store(void* base, long long e) const
    {
        if constexpr (V * sizeof(T) == 16) {
            const uint4 v = Storage<T>::pack(x);
            __builtin_nontemporal_store(tiles::u32x4_t{v.x, v.y, v.z, v.w},
                                        reinterpret_cast<tiles::u32x4_t*>(static_cast<T*>(base) + e));
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) Storage<T>::store1(base, e + i, x[i]);
        }
    }
};

// An item is, in one head of one token: V pairs (half layout: two pieces of V; interleaved: one piece of V, or of one
// pair where V = 1), or, behind the turned channels, a piece that is copied.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    constexpr int U = INTER && V == 1 ? 2 : V;             // elements of a turned piece
    extern __shared__ __align__(16) float2 turn[];         // [tokens][rot / 2] (cos, sin) times m
    const int pairs = a.rot / 2, per = pairs / a.axes;     // pairs of all axes, of one
    const long long first = a.first + static_cast<long long>(blockIdx.x) * a.tokens;
    const int tokens = static_cast<int>(min(static_cast<long long>(a.tokens), static_cast<long long>(a.B) * a.N - first));
    for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
        const int t = fast_div(i, a.div_pairs), p = i - t * pairs;
        const double turns = token_position(a, static_cast<int>(first) + t, p >= per ? 1 : 0) * (a.freqs[p] * 0.15915494309189535);
        const float half_turns = static_cast<float>(2.0 * (turns - rint(turns)));
        float s, c;
        sincospif(half_turns, &s, &c);
        turn[i] = make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
    }
    __syncthreads();
    const int heads = a.t[0].heads + a.t[1].heads, turned = INTER ? a.rot / U : pairs / V;
    const int total = tokens * heads * a.items;
    // kAtOnce items of a thread at a time, all their loads first
    for (int i0 = threadIdx.x; i0 < total; i0 += kAtOnce * kThreads) {
        Piece<T, U> x[kAtOnce], y[kAtOnce];
        const float2* cs[kAtOnce];
        void* to[kAtOnce];
        int it[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = min(i0 + u * kThreads, total - 1);
            const int q = fast_div(i, a.div_items);
            it[u] = i - q * a.items;
            const int t = fast_div(q, a.div_heads), hh = q - t * heads;
            const bool second = hh >= a.t[0].heads;
            const int h = second ? hh - a.t[0].heads : hh;
            const RotaryTensor& e = a.t[second];
            const int token = static_cast<int>(first) + t, b = fast_div(token, a.div_N), n = token - b * a.N;
            const bool copied = it[u] >= turned;
            // (the second axis of the half layout starts at channel 2 per)
            const int p0 = it[u] * V;
            const int c0 = copied ? a.rot + (it[u] - turned) * V : INTER ? it[u] * U : p0 >= per ? p0 + per : p0;
            const T* const from = static_cast<const T*>(e.x) + (b * e.xb + n * e.xn + h * e.xh + c0);
            to[u] = static_cast<T*>(e.y) + (b * e.yb + n * e.yn + h * e.yh + c0);
            cs[u] = turn + t * pairs + (copied ? 0 : INTER ? it[u] * (U / 2) : p0);
            if (INTER && V == 1 && copied) x[u].x[0] = Storage<T>::load1(from, 0);
            else x[u].load(from, 0);
            if (!INTER && !copied) y[u].load(from + per, 0);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (i0 + u * kThreads >= total) break;
            if (it[u] >= turned) {
                if (INTER && V == 1) Storage<T>::store1(to[u], 0, x[u].x[0]);
                else x[u].store(to[u], 0);
            } else if constexpr (INTER) {
#pragma unroll
                for (int j = 0; j < U / 2; ++j) {
                    const float2 w = cs[u][j];
                    const float p = x[u].x[2 * j], q = x[u].x[2 * j + 1];
                    x[u].x[2 * j] = p * w.x - q * w.y;
                    x[u].x[2 * j + 1] = q * w.x + p * w.y;
                }
                x[u].store(to[u], 0);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 w = cs[u][j];
                    const float p = x[u].x[j], q = y[u].x[j];
                    x[u].x[j] = p * w.x - q * w.y;
                    y[u].x[j] = q * w.x + p * w.y;
                }
                x[u].store(to[u], 0);
                y[u].store(static_cast<T*>(to[u]) + per, 0);
            }
        }
    }
}

template <typename T, int V, bool INTER>
hipError_t launch(const RotaryArgs& a, hipStream_t stream)
{
    RotaryArgs p = a;
    constexpr int U = INTER && V == 1 ? 2 : V;
    const int pairs = a.rot / 2, heads = a.t[0].heads + a.t[1].heads;
    p.items = (INTER ? a.rot / U : pairs / V) + (a.d - a.rot) / V;
    // about kAtOnce items a thread, and at most 32 KB of angles
    const long long tokens = static_cast<long long>(a.B) * a.N;
    long long take = (static_cast<long long>(kAtOnce) * kThreads + heads * p.items - 1) / (heads * p.items);
    take = std::min(take, std::max(1LL, 4096LL / std::max(pairs, 1)));
    p.tokens = static_cast<int>(std::max(1LL, std::min(take, tokens)));
    p.div_N = make_fastdiv(a.N);
    p.div_W = make_fastdiv(a.width > 0 ? a.width : 1);
    p.div_pairs = make_fastdiv(std::max(pairs, 1));
    p.div_items = make_fastdiv(p.items);
    p.div_heads = make_fastdiv(heads);
    const long long blocks = (tokens + p.tokens - 1) / p.tokens;
    // HIP takes fewer than 2^32 threads a launch
    constexpr long long most = (1LL << 32) / kThreads - 1;
    for (long long at = 0; at < blocks; at += most) {
        p.first = at * p.tokens;
        hipLaunchKernelGGL((rotary_kernel<T, V, INTER>), dim3(static_cast<unsigned>(std::min(most, blocks - at))), dim3(kThreads),
                           static_cast<size_t>(p.tokens) * pairs * sizeof(float2), stream, p);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const RotaryArgs& a, hipStream_t stream)
{
    // 16-byte pieces where every piece of every row starts on 16 bytes and no piece crosses a border between the
    // halves of an axis, the axes, or the turned and the copied channels; single elements otherwise
    constexpr int V = 16 / static_cast<int>(sizeof(T));
    const int part = a.interleaved ? a.rot : a.rot / a.axes / 2;
    bool wide = part % V == 0 && (a.d - a.rot) % V == 0;
    for (const RotaryTensor& t : a.t) {
        if (t.heads == 0) continue;
        wide = wide && ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.y)) & 15u) == 0;
        for (const long long s : {t.xb, t.xn, t.xh, t.yb, t.yn, t.yh}) wide = wide && s % V == 0;
    }
    if (a.interleaved) return wide ? launch<T, V, true>(a, stream) : launch<T, 1, true>(a, stream);
    return wide ? launch<T, V, false>(a, stream) : launch<T, 1, false>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, bool use_bf16, hipStream_t stream)
{
    return use_bf16 ? launch_type<bf16>(a, stream) : launch_type<float>(a, stream);
}

}  // namespace qta
