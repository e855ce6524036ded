// Group norm with an activation, channels last (the mathematics is in group_norm.h). Bound by memory.
//
// Per token a group's lanes hold its channels in registers, so that everything is read and written once. Maps take two launches that
// each go over them: the first leaves every slab's statistics, the second joins those of its batch element, a few KB, and makes the results.
#include "group_norm.h"
#include "qta_device.h"

namespace qta {
namespace {

constexpr int kT = kNormThreads;


// V elements as they lie in memory, and as numbers.
template <typename T, int V>
struct alignas(V * sizeof(T)) Piece {
    T v[V];
    __device__ __forceinline__ void unpack(float (&x)[V]) const
    {
        if constexpr (V * sizeof(T) == 16) {
            Storage<T>::unpack(__builtin_bit_cast(uint4, *this), x);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = Storage<T>::load1(&v[i], 0);
        }
    }
};
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> piece_at(const void* base, long long e)
{
    return *reinterpret_cast<const Piece<T, V>*>(static_cast<const T*>(base) + e);
}
template <typename T, int V>
__device__ __forceinline__ void load_piece(const void* base, long long e, float (&x)[V])
{
    piece_at<T, V>(base, e).unpack(x);
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(void* base, long long e, const float (&x)[V])
{
    if constexpr (V * sizeof(T) == 16) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, Storage<T>::pack(x)), reinterpret_cast<u32x4*>(static_cast<T*>(base) + e));
    } else {
        Piece<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) Storage<T>::store1(&r.v[i], 0, x[i]);
        *reinterpret_cast<Piece<T, V>*>(static_cast<T*>(base) + e) = r;
    }
}

__device__ __forceinline__ float param(const void* p, bool is_bf16, int c, float otherwise)
{
    if (!p) return otherwise;
    return is_bf16 ? Storage<bf16>::load1(p, c) : Storage<float>::load1(p, c);
}
// N weights from channel c on, or `otherwise`. (One choice for all: a branch for each would wait for each load by itself.)
template <int N>
__device__ __forceinline__ void params(const void* p, bool is_bf16, int c, float otherwise, float (&x)[N])
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = otherwise;
    } else if (is_bf16) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = Storage<bf16>::load1(p, c + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = Storage<float>::load1(p, c + i);
    }
}
__device__ __forceinline__ void store_param(void* p, bool is_bf16, int c, float x)
{
    if (is_bf16) Storage<bf16>::store1(p, c, x);
    else Storage<float>::store1(p, c, x);
}

__device__ __forceinline__ float sigmoid(float z) { return fast_rcp(1.f + __expf(-z)); }
// n values' activations in place, and their slopes. (The choice stands outside the loop: a branch for every value would part the
// instructions of different values.)
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int act)
{
    if (act == QTA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= sigmoid(z[i]);
    } else if (act == QTA_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = 0.5f * z[i] * (1.f + erff(z[i] * 0.70710678118654752f));
    } else if (act == QTA_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] > 0.f ? z[i] : z[i] == z[i] ? 0.f : z[i];
    }
}
template <int N>
__device__ __forceinline__ void slope(float (&z)[N], int act)
{
    if (act == QTA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = sigmoid(z[i]);
            z[i] = s * (1.f + z[i] * (1.f - s));
        }
    } else if (act == QTA_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            z[i] = 0.5f * (1.f + erff(z[i] * 0.70710678118654752f)) + z[i] * __expf(-0.5f * z[i] * z[i]) * 0.39894228040143268f;
    } else if (act == QTA_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] > 0.f ? 1.f : z[i] == z[i] ? 0.f : z[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = 1.f;
    }
}

// The variance, from the mean square of the distances from a rounded mean and their mean, which is what that rounding left. Added to the mean, that
// makes the mean of equal values their value, so that they are nothing but the bias, however large r is. (In one instruction: left * left by itself may
// overflow, and an infinite square less that be no number.)
__device__ __forceinline__ float variance(float square, float left) { return fmaxf(fmaf(-left, left, square), 0.f); }

// Sum over `lanes` (a power of two up to 64) neighbouring lanes, in all of them.
__device__ __forceinline__ float team_sum(float x, int lanes)
{
    if (lanes > 1) x += xchg_f32<1>(x);
    if (lanes > 2) x += xchg_f32<2>(x);
    if (lanes > 4) x += xchg_f32<4>(x);
    if (lanes > 8) x += xchg_f32<8>(x);
    if (lanes > 16) x += xchg_f32<16>(x);
    if (lanes > 32) x += xchg_f32<32>(x);
    return x;
}

// Lanes that a workgroup gives to each of n sums.
__device__ __forceinline__ int team_lanes(int n)
{
    int t = 64;
    while (t > 1 && t * n > kT) t >>= 1;
    return t;
}

// ---- per token ----

template <typename T, int V, int K, bool BACK>
__global__ __launch_bounds__(256) void norm_tokens_kernel(NormArgs a)
{
    const int lane = threadIdx.x & (a.lanes - 1), slot = threadIdx.x / a.lanes;
    const int block = blockIdx.y, row = slot / a.cols, g = block * a.cols + slot - row * a.cols;
    const bool mine = row < a.rows && g < a.groups;
    const int rows = a.B * a.N;
    const float inv = 1.f / a.P;
    float w[K][V], bias[K][V], dw[K][V] = {}, db[K][V] = {};
    bool on[K];
    int at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (lane + k * a.lanes) * V;
        on[k] = mine && c < a.P;
        at[k] = on[k] ? g * a.P + c : 0;
        params(a.weight, a.param_bf16, at[k], 1.f, w[k]);
        params(a.bias, a.param_bf16, at[k], 0.f, bias[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[k][i] = on[k] ? w[k][i] : 0.f;
            bias[k][i] = on[k] ? bias[k][i] : 0.f;
        }
    }
    // (the next token's loads are in flight while one is worked on; rows behind the last are read as that)
    Piece<T, V> px[K], py[K];
    auto fetch = [&](int r0) {
        const int t = min(r0 + (mine ? row : 0), rows - 1), b = fast_div(t, a.div_N);
        const long long from = b * a.xb + (t - b * a.N) * a.xn, to = static_cast<long long>(t) * a.C;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            px[k] = piece_at<T, V>(a.x, from + at[k]);
            if constexpr (BACK) py[k] = piece_at<T, V>(a.dy, to + at[k]);
        }
    };
    const int step = gridDim.x * a.rows;
    fetch(blockIdx.x * a.rows);
    for (int r0 = blockIdx.x * a.rows; r0 < rows; r0 += step) {
        const bool here = mine && r0 + row < rows;
        const long long to = static_cast<long long>(r0 + row) * a.C;
        float x[K][V], dy[K][V];
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            px[k].unpack(x[k]);
            if constexpr (BACK) py[k].unpack(dy[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] = on[k] && here ? x[k][i] : 0.f;
                if constexpr (BACK) dy[k][i] = on[k] && here ? dy[k][i] : 0.f;
                sum += x[k][i];
            }
        }
        if (r0 + step < rows) fetch(r0 + step);
        const float mean = team_sum(sum, a.lanes) * inv;
        float sq = 0.f, left = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] = on[k] ? x[k][i] - mean : 0.f;
                sq += x[k][i] * x[k][i];
                left += x[k][i];
            }
        left = team_sum(left, a.lanes) * inv;
        // (rows behind the last add nothing to the weights' gradients, also where eps is 0)
        const float r = here ? 1.f / sqrtf(variance(team_sum(sq, a.lanes) * inv, left) + a.eps) : 0.f;
        // n = (x - left) r, in one instruction each (places that hold no channel have weights of zero)
        const float shift = -left * r;
        if constexpr (!BACK) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!on[k] || !here) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) x[k][i] = fmaf(x[k][i], r, shift) * w[k][i] + bias[k][i];
                activate(x[k], a.act);
                store_piece<T, V>(a.y, to + at[k], x[k]);
            }
        } else {
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float z[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    x[k][i] = fmaf(x[k][i], r, shift);
                    z[i] = x[k][i] * w[k][i] + bias[k][i];
                }
                slope(z, a.act);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float dz = dy[k][i] * z[i];
                    db[k][i] += dz;
                    dw[k][i] += dz * x[k][i];
                    dy[k][i] = dz * w[k][i];
                    s0 += dy[k][i];
                    s1 += dy[k][i] * x[k][i];
                }
            }
            s0 = team_sum(s0, a.lanes) * inv;
            s1 = team_sum(s1, a.lanes) * inv;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!on[k] || !here) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) x[k][i] = r * (dy[k][i] - s0 - x[k][i] * s1);
                store_piece<T, V>(a.dx, to + at[k], x[k]);
            }
        }
    }
    if constexpr (BACK) {
        if (!a.part) return;
        // rows of the workgroup joined in order
        __shared__ float2 box[256 * V];
        float2* const part = reinterpret_cast<float2*>(a.part) + static_cast<long long>(blockIdx.x) * a.C;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (a.rows > 1) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < V; ++i) box[i * 256 + threadIdx.x] = make_float2(dw[k][i], db[k][i]);
                __syncthreads();
                if (row == 0) {
                    for (int s = 1; s < a.rows; ++s)
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float2 o = box[i * 256 + threadIdx.x + s * a.cols * a.lanes];
                            dw[k][i] += o.x;
                            db[k][i] += o.y;
                        }
                }
            }
            if (row == 0 && on[k]) {
#pragma unroll
                for (int i = 0; i < V; ++i) part[at[k] + i] = make_float2(dw[k][i], db[k][i]);
            }
        }
    }
}

// Sum over a workgroup of 256 threads, in all of them.
__device__ __forceinline__ float group_total(float x, float* box)
{
    x = team_sum(x, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = x;
    __syncthreads();
    return (box[0] + box[1]) + (box[2] + box[3]);
}

// Tokens whose groups no wave holds: a workgroup goes over a group three times (four in the backward), from the second on mostly in
// the caches. Its threads keep the sums of their channels in its row of `part`. Bound by those readings, and in the backward by that row: one group of
// 4096 channels, 16384 tokens in bf16 153 us forward (268 MB) and 677 backward (403 MB), 8192 in fp32 88 and 300.
template <typename T, int V, bool BACK>
__global__ __launch_bounds__(256) void norm_wide_kernel(NormArgs a)
{
    __shared__ float box[4];
    const int g = blockIdx.y, c0 = g * a.P + threadIdx.x * V, c1 = (g + 1) * a.P;
    const int rows = a.B * a.N;
    const float inv = 1.f / a.P;
    float2* const part = a.part ? reinterpret_cast<float2*>(a.part) + static_cast<long long>(blockIdx.x) * a.C : nullptr;
    for (int t = blockIdx.x; t < rows; t += gridDim.x) {
        const int b = fast_div(t, a.div_N);
        const long long from = b * a.xb + (t - b * a.N) * a.xn, to = static_cast<long long>(t) * a.C;
        float x[V], dy[V], sum = 0.f;
        for (int c = c0; c < c1; c += 256 * V) {
            load_piece<T, V>(a.x, from + c, x);
#pragma unroll
            for (int i = 0; i < V; ++i) sum += x[i];
        }
        float mean = group_total(sum, box) * inv, left = 0.f;
        sum = 0.f;
        for (int c = c0; c < c1; c += 256 * V) {
            load_piece<T, V>(a.x, from + c, x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = x[i] - mean;
                sum += d * d;
                left += d;
            }
        }
        left = group_total(left, box) * inv;
        const float r = 1.f / sqrtf(variance(group_total(sum, box) * inv, left) + a.eps);
        mean += left;
        float s0 = 0.f, s1 = 0.f;
        if constexpr (BACK) {
            for (int c = c0; c < c1; c += 256 * V) {
                load_piece<T, V>(a.x, from + c, x);
                load_piece<T, V>(a.dy, to + c, dy);
                float z[V];
#pragma unroll
                for (int i = 0; i < V; ++i)
                    z[i] = (x[i] - mean) * r * param(a.weight, a.param_bf16, c + i, 1.f) + param(a.bias, a.param_bf16, c + i, 0.f);
                slope(z, a.act);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float w = param(a.weight, a.param_bf16, c + i, 1.f), n = (x[i] - mean) * r, dz = dy[i] * z[i];
                    s0 += w * dz;
                    s1 += w * dz * n;
                }
            }
            s0 = group_total(s0, box) * inv;
            s1 = group_total(s1, box) * inv;
        }
        for (int c = c0; c < c1; c += 256 * V) {
            load_piece<T, V>(a.x, from + c, x);
            if constexpr (BACK) load_piece<T, V>(a.dy, to + c, dy);
            float z[V];
#pragma unroll
            for (int i = 0; i < V; ++i)
                z[i] = (x[i] - mean) * r * param(a.weight, a.param_bf16, c + i, 1.f) + param(a.bias, a.param_bf16, c + i, 0.f);
            if constexpr (BACK) {
                slope(z, a.act);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float w = param(a.weight, a.param_bf16, c + i, 1.f), n = (x[i] - mean) * r, dz = dy[i] * z[i];
                    if (part) {
                        const float2 o = t == static_cast<int>(blockIdx.x) ? make_float2(0.f, 0.f) : part[c + i];
                        part[c + i] = make_float2(o.x + dz * n, o.y + dz);
                    }
                    z[i] = r * (w * dz - s0 - n * s1);
                }
            } else {
                activate(z, a.act);
            }
            store_piece<T, V>(BACK ? a.dx : a.y, to + c, z);
        }
    }
}

// ---- maps ----

// Where a workgroup and its threads are.
struct NormPlace {
    int b, slab, block;
    int n0, n1;                 // tokens of the slab
    int row, col;               // of the thread; col is a channel of the tensor
    bool mine;
    int c0, c1;                 // channels of the block
    __device__ __forceinline__ NormPlace(const NormArgs& a, int index, int V)
    {
        block = index % a.blocks;
        const int y = index / a.blocks;
        b = fast_div(y, a.div_slabs);
        slab = y - b * a.slabs;
        n0 = slab * a.slab;
        n1 = min(n0 + a.slab, a.N);
        const int wide = a.cols * V;
        if (a.parts == 1) {
            c0 = block * wide;
            c1 = min(c0 + wide, a.C);
        } else {
            const int g = block / a.parts, p = block - g * a.parts;
            c0 = g * a.P + p * wide;
            c1 = min(c0 + wide, (g + 1) * a.P);
        }
        row = threadIdx.x / a.cols;
        col = c0 + (static_cast<int>(threadIdx.x) - row * a.cols) * V;
        mine = row < a.rows && col < c1;
    }
};

// A thread's tokens of the slab, U at a time, the next ones' loads in flight while these are worked on: before anything else
// (`first`), then work(n, pieces of x, of dy) for each token.
template <typename T, int V, int U, bool DY, bool DOWN>
struct NormStream {
    const T *x, *dy;
    long long xn;
    int C, rows, n, n1, both;
    __device__ __forceinline__ int token(int i) const { return DOWN ? both - i : i; }
    Piece<T, V> px[U], py[DY ? U : 1];
    __device__ __forceinline__ void fetch(int at)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int m = token(min(at + u * rows, n1 - 1));
            px[u] = piece_at<T, V>(x, m * xn);
            if constexpr (DY) py[u] = piece_at<T, V>(dy, static_cast<long long>(m) * C);
        }
    }
    __device__ __forceinline__ NormStream(const NormArgs& a, const NormPlace& at)
        : x(static_cast<const T*>(a.x) + (at.b * a.xb + at.col)), xn(a.xn), C(a.C), rows(a.rows), n(at.mine ? at.n0 + at.row : at.n1), n1(at.n1), both(at.n0 + at.n1 - 1)
    {
        if constexpr (DY) dy = static_cast<const T*>(a.dy) + (static_cast<long long>(at.b) * a.N * a.C + at.col);
        if (n < n1) fetch(n);
    }
    template <typename Work>
    __device__ __forceinline__ void run(Work work)
    {
        for (; n < n1; n += U * rows) {
            float fx[U][V], fy[DY ? U : 1][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                px[u].unpack(fx[u]);
                if constexpr (DY) py[u].unpack(fy[u]);
            }
            if (n + U * rows < n1) fetch(n + U * rows);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (n + u * rows >= n1) break;
                work(token(n + u * rows), fx[u], fy[DY ? u : 0]);
            }
        }
    }
};

// Statistics of a slab: per thread and channel a running mean and sum of squared distances from it; then over the channels and rows of a
// group through LDS, first the mean, then the distances from that.
template <typename T, int V>
__global__ __launch_bounds__(kT) void norm_stats_kernel(NormArgs a)
{
    extern __shared__ __align__(16) float2 box[];                   // [rows][entries of a row]: mean, squares
    const NormPlace at(a, xcd_remap(blockIdx.x, gridDim.x), V);
    float mean[V] = {}, sq[V] = {};
    int count = 0;
    NormStream<T, V, 4, false, false>(a, at).run([&](int, const float (&x)[V], const float (&)[V]) {
        const float inv = fast_rcp(static_cast<float>(++count));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = x[i] - mean[i];
            mean[i] += d * inv;
            sq[i] += d * (x[i] - mean[i]);
        }
    });
    // a thread's channels of one group become one entry
    const bool whole = a.P % V == 0;
    const int each = whole ? 1 : V, wide = a.cols * each, of_group = whole ? min(a.P, at.c1 - at.c0) / V : a.P;
    if (at.mine) {
        float2* const to = box + at.row * wide + (at.col - at.c0) / V * each;
        if (whole) {
            float m = 0.f, left = 0.f, s = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) m += mean[i];
            m *= 1.f / V;
#pragma unroll
            for (int i = 0; i < V; ++i) left += mean[i] - m;
            m += left * (1.f / V);
#pragma unroll
            for (int i = 0; i < V; ++i) s += sq[i] + count * (mean[i] - m) * (mean[i] - m);
            to[0] = make_float2(m, s);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) to[i] = make_float2(mean[i], sq[i]);
        }
    }
    __syncthreads();
    const int groups = a.parts == 1 ? (at.c1 - at.c0) / a.P : 1, lanes = team_lanes(groups), tokens = at.n1 - at.n0;
    const int lane = threadIdx.x & (lanes - 1);
    const float per = static_cast<float>(whole ? V : 1);
    for (int g = threadIdx.x / lanes; g < groups; g += kT / lanes) {
        float m = 0.f, left = 0.f, s = 0.f;
        const float entries = static_cast<float>(tokens) * of_group;
        // (a part of a group is wider than half a workgroup: one row)
        auto each = [&](auto add) {
#pragma unroll 4
            for (int i = lane; i < a.rows * of_group; i += lanes) {
                const int r = a.rows == 1 ? 0 : fast_div(i, a.div_entry);
                add(box[r * (wide - of_group) + g * of_group + i], static_cast<float>(fast_div(tokens - r + a.rows - 1, a.div_rows)));
            }
        };
        each([&](float2 v, float n) { m += n * v.x; });
        m = team_sum(m, lanes) / entries;
        each([&](float2 v, float n) {
            const float d = v.x - m;
            left += n * d;
            s += v.y + n * per * d * d;
        });
        left = team_sum(left, lanes) / entries;
        s = entries * per * variance(team_sum(s, lanes) / (entries * per), left);
        m += left;
        const int entry = a.parts == 1 ? at.c0 / a.P + g : at.block;
        if (lane == 0) reinterpret_cast<float2*>(a.part)[(static_cast<long long>(at.b) * a.slabs + at.slab) * a.entries + entry] = make_float2(m, s);
    }
}

// What the slabs (and a group's parts) left for one group, spread over a team's lanes: add(entry, slab, part).
template <typename Add>
__device__ __forceinline__ void each_entry(const NormArgs& a, const float2* from, int lane, int lanes, Add add)
{
    if (a.parts == 1) {
#pragma unroll 8
        for (int s = lane; s < a.slabs; s += lanes) add(from[s * a.entries], s, 0);
    } else {
        for (int i = lane; i < a.slabs * a.parts; i += lanes) {
            const int s = i / a.parts, p = i - s * a.parts;
            add(from[s * a.entries + p], s, p);
        }
    }
}

// Mean and r of a block's groups, from the slabs' statistics, into LDS.
__device__ __forceinline__ void join_stats(const NormArgs& a, const NormPlace& at, int V, float2* box)
{
    const int g0 = at.c0 / a.P, groups = a.parts == 1 ? (at.c1 - at.c0) / a.P : 1, lanes = team_lanes(groups);
    const int lane = threadIdx.x & (lanes - 1);
    const float2* const part = reinterpret_cast<const float2*>(a.part) + static_cast<long long>(at.b) * a.slabs * a.entries;
    const float inv = 1.f / (static_cast<float>(a.N) * a.P);
    for (int g = threadIdx.x / lanes; g < groups; g += kT / lanes) {
        const float2* const from = part + (g0 + g) * a.parts;
        // the mean, then the distances from it, as in a slab. A lane's first entries stay in registers between the two (2 x 19200 tokens of 256 channels, bf16: a pass takes 17.4 us, with them read again 18.9, before the means were corrected)
        constexpr int kHeld = 8;
        const int total = a.slabs * a.parts;
        auto fetch = [&](int i, float2& v, float& n) {
            const int slab = a.parts == 1 ? i : i / a.parts, p = i - slab * a.parts;
            v = from[static_cast<long long>(slab) * a.entries + p];
            n = static_cast<float>(min(a.slab, a.N - slab * a.slab)) * (a.parts == 1 ? a.P : min(a.cols * V, a.P - p * a.cols * V));
        };
        float2 held[kHeld];
        float counts[kHeld];
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            held[u] = make_float2(0.f, 0.f);
            counts[u] = 0.f;
            if (lane + u * lanes < total) fetch(lane + u * lanes, held[u], counts[u]);
        }
        auto each = [&](auto add) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u) add(held[u], counts[u]);
            for (int i = lane + kHeld * lanes; i < total; i += lanes) {
                float2 v;
                float n;
                fetch(i, v, n);
                add(v, n);
            }
        };
        float m = 0.f, left = 0.f, s = 0.f;
        each([&](float2 v, float n) { m += n * v.x; });
        m = team_sum(m, lanes) * inv;
        each([&](float2 v, float n) {
            const float d = v.x - m;
            left += n * d;
            s += v.y + n * d * d;
        });
        left = team_sum(left, lanes) * inv;
        const float r = 1.f / sqrtf(variance(team_sum(s, lanes) * inv, left) + a.eps);
        m += left;
        if (lane == 0) {
            box[g] = make_float2(m, r);
            if (a.stats && at.slab == 0 && (a.parts == 1 || at.block % a.parts == 0))
                reinterpret_cast<float2*>(a.stats)[static_cast<long long>(at.b) * a.groups + g0 + g] = make_float2(m, r);
        }
    }
    __syncthreads();
}

template <typename T, int V>
__global__ __launch_bounds__(kT) void norm_apply_kernel(NormArgs a)
{
    extern __shared__ __align__(16) float2 box[];
    const NormPlace at(a, xcd_remap(blockIdx.x, gridDim.x), V);
    NormStream<T, V, 4, false, true> stream(a, at);
    float f[V], bias[V];
    params(a.weight, a.param_bf16, at.mine ? at.col : 0, 1.f, f);
    params(a.bias, a.param_bf16, at.mine ? at.col : 0, 0.f, bias);
    join_stats(a, at, V, box);
    if (!at.mine) return;
    float mean[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = box[fast_div(at.col + i, a.div_P) - at.c0 / a.P];
        mean[i] = s.x;
        f[i] *= s.y;
    }
    const long long to = static_cast<long long>(at.b) * a.N * a.C + at.col;
    stream.run([&](int n, const float (&x)[V], const float (&)[V]) {
        float z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = (x[i] - mean[i]) * f[i] + bias[i];
        activate(z, a.act);
        store_piece<T, V>(a.y, to + static_cast<long long>(n) * a.C, z);
    });
}

// A thread's channels in the backward.
template <int V>
struct NormChannels {
    float mean[V], r[V], w[V], bias[V];
    __device__ __forceinline__ NormChannels(const NormArgs& a, const NormPlace& at)
    {
        params(a.weight, a.param_bf16, at.mine ? at.col : 0, 1.f, w);
        params(a.bias, a.param_bf16, at.mine ? at.col : 0, 0.f, bias);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 s = reinterpret_cast<const float2*>(a.stats)[static_cast<long long>(at.b) * a.groups + (at.mine ? fast_div(at.col + i, a.div_P) : 0)];
            mean[i] = s.x;
            r[i] = s.y;
        }
    }
};

// Sums over a slab's tokens of dz n and dz for every channel.
template <typename T, int V>
__global__ __launch_bounds__(kT) void norm_sums_kernel(NormArgs a)
{
    extern __shared__ __align__(16) float2 box[];                   // [V][kT]
    const NormPlace at(a, xcd_remap(blockIdx.x, gridDim.x), V);
    NormStream<T, V, 2, true, false> stream(a, at);
    float s1[V] = {}, s0[V] = {}, f[V];
    const NormChannels<V> ch(a, at);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = ch.r[i] * ch.w[i];
    stream.run([&](int, const float (&x)[V], const float (&dy)[V]) {
        float d[V], z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            d[i] = x[i] - ch.mean[i];
            z[i] = d[i] * f[i] + ch.bias[i];
        }
        slope(z, a.act);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float dz = dy[i] * z[i];
            s1[i] += dz * d[i];
            s0[i] += dz;
        }
    });
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] *= ch.r[i];
#pragma unroll
    for (int i = 0; i < V; ++i) box[i * kT + threadIdx.x] = make_float2(s1[i], s0[i]);
    __syncthreads();
    // rows of a channel: a team of lanes each
    const long long slab = static_cast<long long>(at.b) * a.slabs + at.slab;
    float2* const part = reinterpret_cast<float2*>(a.part) + slab * a.C;
    const int wide = at.c1 - at.c0, team = min(team_lanes(wide), a.rows_lanes), of = threadIdx.x & (team - 1);
    for (int c = threadIdx.x / team; c < wide; c += kT / team) {
        const int col = c / V, i = c - col * V;
        float2 s = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int r = of; r < a.rows; r += team) {
            const float2 o = box[i * kT + col + r * a.cols];
            s.x += o.x;
            s.y += o.y;
        }
        s.x = team_sum(s.x, team);
        s.y = team_sum(s.y, team);
        // (a channel's first row is its team's alone to read)
        if (of == 0) {
            box[i * kT + col] = s;
            part[at.c0 + c] = s;
        }
    }
    __syncthreads();
    const int groups = a.parts == 1 ? wide / a.P : 1, lanes = team_lanes(groups), lane = threadIdx.x & (lanes - 1);
    const int of_group = a.parts == 1 ? a.P : wide;
    for (int g = threadIdx.x / lanes; g < groups; g += kT / lanes) {
        float t1 = 0.f, t0 = 0.f;
        for (int i = lane; i < of_group; i += lanes) {
            const int c = g * of_group + i, col = c / V;
            const float2 o = box[(c - col * V) * kT + col];
            const float w = param(a.weight, a.param_bf16, at.c0 + c, 1.f);
            t1 += w * o.x;
            t0 += w * o.y;
        }
        t1 = team_sum(t1, lanes);
        t0 = team_sum(t0, lanes);
        const int entry = a.parts == 1 ? at.c0 / a.P + g : at.block;
        if (lane == 0) reinterpret_cast<float2*>(a.group_part)[slab * a.entries + entry] = make_float2(t1, t0);
    }
}

// Gradients of the weights: sums of the workgroups' sums, 16 channels a workgroup.
__device__ __forceinline__ void norm_params(const NormArgs& a, int block, int threads, float2* box)
{
    const int c = block * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4, slices = threads / 16;
    const float2* const part = reinterpret_cast<const float2*>(a.part);
    float2 s = make_float2(0.f, 0.f);
    if (c < a.C) {
        const int n0 = static_cast<int>(static_cast<long long>(a.sums) * slice / slices), n1 = static_cast<int>(static_cast<long long>(a.sums) * (slice + 1) / slices);
        for (int n = n0; n < n1; n += 4) {
            float2 o[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] = part[static_cast<long long>(min(n + u, n1 - 1)) * a.C + c];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (n + u >= n1) break;
                s.x += o[u].x;
                s.y += o[u].y;
            }
        }
    }
    s.x += xchg_f32<16>(s.x);
    s.y += xchg_f32<16>(s.y);
    s.x += xchg_f32<32>(s.x);
    s.y += xchg_f32<32>(s.y);
    if ((threadIdx.x & 63) < 16) box[(threadIdx.x >> 6) * 16 + (threadIdx.x & 15)] = s;
    __syncthreads();
    if (slice == 0 && c < a.C) {
#pragma unroll 4
        for (int i = 1; i < threads / 64; ++i) {
            s.x += box[i * 16 + threadIdx.x].x;
            s.y += box[i * 16 + threadIdx.x].y;
        }
        if (a.dweight) store_param(a.dweight, a.param_bf16, c, s.x);
        if (a.dbias) store_param(a.dbias, a.param_bf16, c, s.y);
    }
}
__global__ __launch_bounds__(kT) void norm_params_kernel(NormArgs a)
{
    __shared__ float2 box[kT];
    norm_params(a, blockIdx.x, kT, box);
}

// dx, from the sums of its batch element's slabs; the last workgroups make the gradients of the weights.
template <typename T, int V>
__global__ __launch_bounds__(kT) void norm_dx_kernel(NormArgs a)
{
    extern __shared__ __align__(16) float2 box[];
    const int own = static_cast<int>(a.own);
    if (static_cast<int>(blockIdx.x) >= own) return norm_params(a, blockIdx.x - own, kT, box);
    const NormPlace at(a, xcd_remap(blockIdx.x, own), V);
    NormStream<T, V, 2, true, true> stream(a, at);
    const NormChannels<V> ch(a, at);
    const int g0 = at.c0 / a.P, groups = a.parts == 1 ? (at.c1 - at.c0) / a.P : 1, lanes = team_lanes(groups);
    const int lane = threadIdx.x & (lanes - 1);
    const float2* const part = reinterpret_cast<const float2*>(a.group_part) + static_cast<long long>(at.b) * a.slabs * a.entries;
    const float inv = 1.f / (static_cast<float>(a.N) * a.P);
    for (int g = threadIdx.x / lanes; g < groups; g += kT / lanes) {
        float s1 = 0.f, s0 = 0.f;
        each_entry(a, part + (g0 + g) * a.parts, lane, lanes, [&](float2 v, int, int) {
            s1 += v.x;
            s0 += v.y;
        });
        s1 = team_sum(s1, lanes) * inv;
        s0 = team_sum(s0, lanes) * inv;
        if (lane == 0) box[g] = make_float2(s1, s0);
    }
    __syncthreads();
    if (!at.mine) return;
    float s1[V], s0[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = box[fast_div(at.col + i, a.div_P) - g0];
        s1[i] = s.x;
        s0[i] = s.y;
    }
    const long long to = static_cast<long long>(at.b) * a.N * a.C + at.col;
    stream.run([&](int t, const float (&x)[V], const float (&dy)[V]) {
        float n[V], z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            n[i] = (x[i] - ch.mean[i]) * ch.r[i];
            z[i] = n[i] * ch.w[i] + ch.bias[i];
        }
        slope(z, a.act);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = ch.r[i] * (dy[i] * z[i] * ch.w[i] - s0[i] - n[i] * s1[i]);
        store_piece<T, V>(a.dx, to + static_cast<long long>(t) * a.C, z);
    });
}

template <typename T, int V, bool BACK>
void launch_tokens(const NormArgs& a, const NormPlan& p, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(p.grid), static_cast<unsigned>(p.blocks));
    if (p.wide) hipLaunchKernelGGL((norm_wide_kernel<T, V, BACK>), grid, dim3(256), 0, stream, a);
    else if (p.pieces == 1) hipLaunchKernelGGL((norm_tokens_kernel<T, V, 1, BACK>), grid, dim3(256), 0, stream, a);
    else if (p.pieces == 2) hipLaunchKernelGGL((norm_tokens_kernel<T, V, 2, BACK>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((norm_tokens_kernel<T, V, 4, BACK>), grid, dim3(256), 0, stream, a);
}

template <typename T, int V>
hipError_t launch(NormArgs a, const NormPlan& p, bool back, hipStream_t stream)
{
    a.cols = p.cols;
    a.rows = p.rows;
    a.slabs = p.slabs;
    a.slab = p.slab;
    a.div_rows = make_fastdiv(p.rows);
    a.div_entry = make_fastdiv(a.P % V == 0 ? a.P / V : a.P);
    a.rows_lanes = 1;
    while (a.rows_lanes < p.rows && a.rows_lanes < 64) a.rows_lanes *= 2;
    a.group_part = a.part ? a.part + p.channel_floats : nullptr;
    a.div_slabs = make_fastdiv(std::max(p.slabs, 1));
    a.blocks = p.blocks;
    a.parts = p.parts;
    a.lanes = p.lanes;
    a.div_N = make_fastdiv(a.N);
    a.div_P = make_fastdiv(a.P);
    const unsigned param_blocks = a.dweight || a.dbias ? static_cast<unsigned>((a.C + 15) / 16) : 0;
    if (p.tokens) {
        a.sums = p.grid;
        if (!back) launch_tokens<T, V, false>(a, p, stream);
        else launch_tokens<T, V, true>(a, p, stream);
        if (back && param_blocks) hipLaunchKernelGGL(norm_params_kernel, dim3(param_blocks), dim3(kT), 0, stream, a);
        return hipGetLastError();
    }
    a.entries = a.groups * p.parts;
    a.sums = a.B * p.slabs;
    const size_t groups_lds = static_cast<size_t>(p.parts == 1 ? std::max(1, std::min(a.groups, p.cols * V / a.P)) : 1) * sizeof(float2);
    const size_t entries_lds = static_cast<size_t>(p.rows) * p.cols * (a.P % V == 0 ? 1 : V) * sizeof(float2);
    const unsigned grid = a.own = static_cast<unsigned>(a.B) * p.slabs * p.blocks;
    if (!back) {
        hipLaunchKernelGGL((norm_stats_kernel<T, V>), dim3(grid), dim3(kT), entries_lds, stream, a);
        hipLaunchKernelGGL((norm_apply_kernel<T, V>), dim3(grid), dim3(kT), groups_lds, stream, a);
    } else {
        hipLaunchKernelGGL((norm_sums_kernel<T, V>), dim3(grid), dim3(kT), static_cast<size_t>(kT) * V * sizeof(float2), stream, a);
        hipLaunchKernelGGL((norm_dx_kernel<T, V>), dim3(grid + param_blocks), dim3(kT), std::max(groups_lds, kT * sizeof(float2)), stream, a);
    }
    return hipGetLastError();
}

hipError_t launch_type(const NormArgs& a, const NormPlan& p, bool use_bf16, bool back, hipStream_t stream)
{
    if (use_bf16) {
        if (p.V == 8) return launch<bf16, 8>(a, p, back, stream);
        if (p.V == 4) return launch<bf16, 4>(a, p, back, stream);
        return p.V == 2 ? launch<bf16, 2>(a, p, back, stream) : launch<bf16, 1>(a, p, back, stream);
    }
    if (p.V == 4) return launch<float, 4>(a, p, back, stream);
    return p.V == 2 ? launch<float, 2>(a, p, back, stream) : launch<float, 1>(a, p, back, stream);
}

}  // namespace

hipError_t launch_norm_forward(const NormArgs& a, const NormPlan& p, bool use_bf16, hipStream_t stream)
{
    return launch_type(a, p, use_bf16, false, stream);
}

hipError_t launch_norm_backward(const NormArgs& a, const NormPlan& p, bool use_bf16, hipStream_t stream)
{
    return launch_type(a, p, use_bf16, true, stream);
}

}  // namespace qta
