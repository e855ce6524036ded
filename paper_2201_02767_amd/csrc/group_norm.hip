// Group norm with an activation, channels last (the mathematics is in group_norm.h). Bound by memory.
//
// Per token a group's lanes hold its channels in registers, so that everything is read and written once. Maps take two launches that
// each go over them: the first leaves every slab's statistics, the second joins those of its batch element, a few KB, and makes the results.
#include "group_norm.h"
#include "qta_device.h"

namespace qta {
namespace {

constexpr int kT = kNormThreads;

// V elements at element e.
template <typename T, int V>
__device__ __forceinline__ void load_piece(const void* base, long long e, float (&x)[V])
{
    if constexpr (V * sizeof(T) == 16) {
        Storage<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(base) + e), x);
    } else {
        struct alignas(V * sizeof(T)) Raw { T v[V]; };
        const Raw r = *reinterpret_cast<const Raw*>(static_cast<const T*>(base) + e);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = Storage<T>::load1(&r.v[i], 0);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(void* base, long long e, const float (&x)[V])
{
    if constexpr (V * sizeof(T) == 16) {
        *reinterpret_cast<uint4*>(static_cast<T*>(base) + e) = Storage<T>::pack(x);
    } else {
        struct alignas(V * sizeof(T)) Raw { T v[V]; };
        Raw r;
#pragma unroll
        for (int i = 0; i < V; ++i) Storage<T>::store1(&r.v[i], 0, x[i]);
        *reinterpret_cast<Raw*>(static_cast<T*>(base) + e) = r;
    }
}

__device__ __forceinline__ float param(const void* p, bool is_bf16, int c, float otherwise)
{
    if (!p) return otherwise;
    return is_bf16 ? Storage<bf16>::load1(p, c) : Storage<float>::load1(p, c);
}
__device__ __forceinline__ void store_param(void* p, bool is_bf16, int c, float x)
{
    if (is_bf16) Storage<bf16>::store1(p, c, x);
    else Storage<float>::store1(p, c, x);
}

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + __expf(-z)); }
__device__ __forceinline__ float activate(float z, int act)
{
    if (act == QTA_ACT_SILU) return z * sigmoid(z);
    if (act == QTA_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    if (act == QTA_ACT_RELU) return z > 0.f ? z : z == z ? 0.f : z;
    return z;
}
__device__ __forceinline__ float slope(float z, int act)
{
    if (act == QTA_ACT_SILU) {
        const float s = sigmoid(z);
        return s * (1.f + z * (1.f - s));
    }
    if (act == QTA_ACT_GELU) return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    if (act == QTA_ACT_RELU) return z > 0.f ? 1.f : z == z ? 0.f : z;
    return 1.f;
}

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
    const long long rows = static_cast<long long>(a.B) * a.N;
    const float inv = 1.f / a.P;
    float w[K][V], bias[K][V], dw[K][V] = {}, db[K][V] = {};
    bool on[K];
    int at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (lane + k * a.lanes) * V;
        on[k] = mine && c < a.P;
        at[k] = on[k] ? g * a.P + c : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[k][i] = on[k] ? param(a.weight, a.param_bf16, at[k] + i, 1.f) : 0.f;
            bias[k][i] = on[k] ? param(a.bias, a.param_bf16, at[k] + i, 0.f) : 0.f;
        }
    }
    for (long long r0 = static_cast<long long>(blockIdx.x) * a.rows; r0 < rows; r0 += static_cast<long long>(gridDim.x) * a.rows) {
        const long long t = r0 + row;
        const bool here = mine && t < rows;
        const int tt = static_cast<int>(here ? t : r0), b = fast_div(tt, a.div_N);
        const long long from = b * a.xb + (tt - b * a.N) * a.xn, to = static_cast<long long>(tt) * a.C;
        float x[K][V], dy[K][V];
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (on[k] && here) {
                load_piece<T, V>(a.x, from + at[k], x[k]);
                if constexpr (BACK) load_piece<T, V>(a.dy, to + at[k], dy[k]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) x[k][i] = dy[k][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum += x[k][i];
        }
        const float mean = team_sum(sum, a.lanes) * inv;
        float sq = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] = on[k] ? x[k][i] - mean : 0.f;
                sq += x[k][i] * x[k][i];
            }
        // (rows behind the last add nothing to the weights' gradients, also where eps is 0)
        const float r = here ? 1.f / sqrtf(team_sum(sq, a.lanes) * inv + a.eps) : 0.f;
        if constexpr (!BACK) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!on[k] || !here) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) x[k][i] = activate(x[k][i] * r * w[k][i] + bias[k][i], a.act);
                store_piece<T, V>(a.y, to + at[k], x[k]);
            }
        } else {
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    x[k][i] *= r;
                    const float dz = dy[k][i] * slope(x[k][i] * w[k][i] + bias[k][i], a.act);
                    db[k][i] += dz;
                    dw[k][i] += dz * x[k][i];
                    dy[k][i] = dz * w[k][i];
                    s0 += dy[k][i];
                    s1 += dy[k][i] * x[k][i];
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
// the caches. Its threads keep the sums of their channels in its row of `part`.
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
        const float mean = group_total(sum, box) * inv;
        sum = 0.f;
        for (int c = c0; c < c1; c += 256 * V) {
            load_piece<T, V>(a.x, from + c, x);
#pragma unroll
            for (int i = 0; i < V; ++i) sum += (x[i] - mean) * (x[i] - mean);
        }
        const float r = 1.f / sqrtf(group_total(sum, box) * inv + a.eps);
        float s0 = 0.f, s1 = 0.f;
        if constexpr (BACK) {
            for (int c = c0; c < c1; c += 256 * V) {
                load_piece<T, V>(a.x, from + c, x);
                load_piece<T, V>(a.dy, to + c, dy);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float w = param(a.weight, a.param_bf16, c + i, 1.f), n = (x[i] - mean) * r;
                    const float dz = dy[i] * slope(n * w + param(a.bias, a.param_bf16, c + i, 0.f), a.act);
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
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float w = param(a.weight, a.param_bf16, c + i, 1.f), n = (x[i] - mean) * r;
                const float z = n * w + param(a.bias, a.param_bf16, c + i, 0.f);
                if constexpr (BACK) {
                    const float dz = dy[i] * slope(z, a.act);
                    if (part) {
                        const float2 o = t == static_cast<int>(blockIdx.x) ? make_float2(0.f, 0.f) : part[c + i];
                        part[c + i] = make_float2(o.x + dz * n, o.y + dz);
                    }
                    x[i] = r * (w * dz - s0 - n * s1);
                } else {
                    x[i] = activate(z, a.act);
                }
            }
            store_piece<T, V>(BACK ? a.dx : a.y, to + c, x);
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
        b = y / a.slabs;
        slab = y - b * a.slabs;
        n0 = static_cast<int>(static_cast<long long>(a.N) * slab / a.slabs);
        n1 = static_cast<int>(static_cast<long long>(a.N) * (slab + 1) / a.slabs);
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

// Statistics of a slab: per thread and channel a running mean and sum of squared distances from it; then over the channels and rows of a
// group through LDS, first the mean, then the distances from that.
template <typename T, int V>
__global__ __launch_bounds__(kT) void norm_stats_kernel(NormArgs a)
{
    constexpr int U = 4;                                            // tokens whose loads are in flight
    extern __shared__ __align__(16) float2 box[];                   // [rows][entries of a row]: mean, squares
    const NormPlace at(a, xcd_remap(blockIdx.x, gridDim.x), V);
    float mean[V] = {}, sq[V] = {};
    int count = 0;
    if (at.mine) {
        const long long from = at.b * a.xb + at.col;
        for (int n = at.n0 + at.row; n < at.n1; n += U * a.rows) {
            float x[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) load_piece<T, V>(a.x, from + min(n + u * a.rows, at.n1 - 1) * a.xn, x[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (n + u * a.rows >= at.n1) break;
                const float inv = fast_rcp(static_cast<float>(++count));
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = x[u][i] - mean[i];
                    mean[i] += d * inv;
                    sq[i] += d * (x[u][i] - mean[i]);
                }
            }
        }
    }
    // a thread's channels of one group become one entry
    const bool whole = a.P % V == 0;
    const int each = whole ? 1 : V, wide = a.cols * each, of_group = whole ? min(a.P, at.c1 - at.c0) / V : a.P;
    if (at.mine) {
        float2* const to = box + at.row * wide + (at.col - at.c0) / V * each;
        if (whole) {
            float m = 0.f, s = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) m += mean[i];
            m *= 1.f / V;
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
        float m = 0.f, s = 0.f;
        for (int r = 0; r < a.rows; ++r) {
            const float n = static_cast<float>((tokens - r + a.rows - 1) / a.rows);
            for (int e = lane; e < of_group; e += lanes) m += n * box[r * wide + g * of_group + e].x;
        }
        m = team_sum(m, lanes) / (static_cast<float>(tokens) * of_group);
        for (int r = 0; r < a.rows; ++r) {
            const float n = static_cast<float>((tokens - r + a.rows - 1) / a.rows) * per;
            for (int e = lane; e < of_group; e += lanes) {
                const float2 v = box[r * wide + g * of_group + e];
                s += v.y + n * (v.x - m) * (v.x - m);
            }
        }
        s = team_sum(s, lanes);
        const int entry = a.parts == 1 ? at.c0 / a.P + g : at.block;
        if (lane == 0) reinterpret_cast<float2*>(a.part)[(static_cast<long long>(at.b) * a.slabs + at.slab) * a.entries + entry] = make_float2(m, s);
    }
}

// Mean and r of a block's groups, from the slabs' statistics, into LDS.
__device__ __forceinline__ void join_stats(const NormArgs& a, const NormPlace& at, int V, float2* box)
{
    const int g0 = at.c0 / a.P, groups = a.parts == 1 ? (at.c1 - at.c0) / a.P : 1, lanes = team_lanes(groups);
    const int lane = threadIdx.x & (lanes - 1), n = a.slabs * a.parts;
    const float2* const part = reinterpret_cast<const float2*>(a.part) + static_cast<long long>(at.b) * a.slabs * a.entries;
    const float inv = 1.f / (static_cast<float>(a.N) * a.P);
    // values of part p of slab s
    auto values = [&](int s, int p) {
        const int tokens = static_cast<int>(static_cast<long long>(a.N) * (s + 1) / a.slabs) - static_cast<int>(static_cast<long long>(a.N) * s / a.slabs);
        return static_cast<float>(tokens) * (a.parts == 1 ? a.P : min(a.cols * V, a.P - p * a.cols * V));
    };
    for (int g = threadIdx.x / lanes; g < groups; g += kT / lanes) {
        float m = 0.f, s = 0.f;
        for (int i = lane; i < n; i += lanes) {
            const int slab = i / a.parts, p = i - slab * a.parts;
            m += values(slab, p) * part[slab * a.entries + (g0 + g) * a.parts + p].x;
        }
        m = team_sum(m, lanes) * inv;
        for (int i = lane; i < n; i += lanes) {
            const int slab = i / a.parts, p = i - slab * a.parts;
            const float2 v = part[slab * a.entries + (g0 + g) * a.parts + p];
            s += v.y + values(slab, p) * (v.x - m) * (v.x - m);
        }
        const float r = 1.f / sqrtf(team_sum(s, lanes) * inv + a.eps);
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
    constexpr int U = 4;
    extern __shared__ __align__(16) float2 box[];
    const NormPlace at(a, xcd_remap(blockIdx.x, gridDim.x), V);
    join_stats(a, at, V, box);
    if (!at.mine) return;
    float mean[V], f[V], bias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = box[(at.col + i) / a.P - at.c0 / a.P];
        mean[i] = s.x;
        f[i] = s.y * param(a.weight, a.param_bf16, at.col + i, 1.f);
        bias[i] = param(a.bias, a.param_bf16, at.col + i, 0.f);
    }
    const long long from = at.b * a.xb + at.col, to = static_cast<long long>(at.b) * a.N * a.C + at.col;
    for (int n = at.n0 + at.row; n < at.n1; n += U * a.rows) {
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load_piece<T, V>(a.x, from + min(n + u * a.rows, at.n1 - 1) * a.xn, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n + u * a.rows >= at.n1) break;
#pragma unroll
            for (int i = 0; i < V; ++i) x[u][i] = activate((x[u][i] - mean[i]) * f[i] + bias[i], a.act);
            store_piece<T, V>(a.y, to + static_cast<long long>(n + u * a.rows) * a.C, x[u]);
        }
    }
}

// A thread's channels in the backward.
template <int V>
struct NormChannels {
    float mean[V], r[V], w[V], bias[V];
    __device__ __forceinline__ NormChannels(const NormArgs& a, const NormPlace& at)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 s = reinterpret_cast<const float2*>(a.stats)[static_cast<long long>(at.b) * a.groups + (at.mine ? (at.col + i) / a.P : 0)];
            mean[i] = s.x;
            r[i] = s.y;
            w[i] = param(a.weight, a.param_bf16, at.mine ? at.col + i : 0, 1.f);
            bias[i] = param(a.bias, a.param_bf16, at.mine ? at.col + i : 0, 0.f);
        }
    }
};

// Sums over a slab's tokens of dz n and dz for every channel.
template <typename T, int V>
__global__ __launch_bounds__(kT) void norm_sums_kernel(NormArgs a)
{
    constexpr int U = 2;
    extern __shared__ __align__(16) float2 box[];                   // [V][kT]
    const NormPlace at(a, xcd_remap(blockIdx.x, gridDim.x), V);
    float s1[V] = {}, s0[V] = {};
    if (at.mine) {
        const NormChannels<V> ch(a, at);
        const long long from = at.b * a.xb + at.col, up = static_cast<long long>(at.b) * a.N * a.C + at.col;
        for (int n = at.n0 + at.row; n < at.n1; n += U * a.rows) {
            float x[U][V], dy[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int m = min(n + u * a.rows, at.n1 - 1);
                load_piece<T, V>(a.x, from + m * a.xn, x[u]);
                load_piece<T, V>(a.dy, up + static_cast<long long>(m) * a.C, dy[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (n + u * a.rows >= at.n1) break;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float v = (x[u][i] - ch.mean[i]) * ch.r[i], dz = dy[u][i] * slope(v * ch.w[i] + ch.bias[i], a.act);
                    s1[i] += dz * v;
                    s0[i] += dz;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) box[i * kT + threadIdx.x] = make_float2(s1[i], s0[i]);
    __syncthreads();
    float2* const part = reinterpret_cast<float2*>(a.part) + (static_cast<long long>(at.b) * a.slabs + at.slab) * a.C;
    const int wide = (at.c1 - at.c0);
    for (int c = threadIdx.x; c < wide; c += kT) {
        const int col = c / V, i = c - col * V;
        float2 s = box[i * kT + col];
        for (int r = 1; r < a.rows; ++r) {
            const float2 o = box[i * kT + col + r * a.cols];
            s.x += o.x;
            s.y += o.y;
        }
        part[at.c0 + c] = s;
    }
}

// Gradients of the weights: sums of the workgroups' sums, 32 channels a workgroup.
__device__ __forceinline__ void norm_params(const NormArgs& a, int block, int threads, float2* box)
{
    const int c = block * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, slices = threads / 32;
    const float2* const part = reinterpret_cast<const float2*>(a.part);
    float2 s = make_float2(0.f, 0.f);
    if (c < a.C) {
        const int n0 = static_cast<int>(static_cast<long long>(a.sums) * slice / slices), n1 = static_cast<int>(static_cast<long long>(a.sums) * (slice + 1) / slices);
        for (int n = n0; n < n1; n += 8) {
            float2 o[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = part[static_cast<long long>(min(n + u, n1 - 1)) * a.C + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (n + u >= n1) break;
                s.x += o[u].x;
                s.y += o[u].y;
            }
        }
    }
    box[threadIdx.x] = s;
    __syncthreads();
    if (slice == 0 && c < a.C) {
        for (int i = 1; i < slices; ++i) {
            s.x += box[i * 32 + threadIdx.x].x;
            s.y += box[i * 32 + threadIdx.x].y;
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
    constexpr int U = 2;
    extern __shared__ __align__(16) float2 box[];
    const int own = a.B * a.slabs * a.blocks;
    if (static_cast<int>(blockIdx.x) >= own) return norm_params(a, blockIdx.x - own, kT, box);
    const NormPlace at(a, xcd_remap(blockIdx.x, own), V);
    const int g0 = at.c0 / a.P, groups = a.parts == 1 ? (at.c1 - at.c0) / a.P : 1, lanes = team_lanes(groups);
    const int lane = threadIdx.x & (lanes - 1);
    const float2* const part = reinterpret_cast<const float2*>(a.part) + static_cast<long long>(at.b) * a.slabs * a.C;
    const float inv = 1.f / (static_cast<float>(a.N) * a.P);
    for (int g = threadIdx.x / lanes; g < groups; g += kT / lanes) {
        float s1 = 0.f, s0 = 0.f;
#pragma unroll 4
        for (int i = lane; i < a.slabs * a.P; i += lanes) {
            const int slab = fast_div(i, a.div_P), c = (g0 + g) * a.P + i - slab * a.P;
            const float w = param(a.weight, a.param_bf16, c, 1.f);
            const float2 o = part[static_cast<long long>(slab) * a.C + c];
            s1 += w * o.x;
            s0 += w * o.y;
        }
        s1 = team_sum(s1, lanes) * inv;
        s0 = team_sum(s0, lanes) * inv;
        if (lane == 0) box[g] = make_float2(s1, s0);
    }
    __syncthreads();
    if (!at.mine) return;
    const NormChannels<V> ch(a, at);
    float s1[V], s0[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = box[(at.col + i) / a.P - g0];
        s1[i] = s.x;
        s0[i] = s.y;
    }
    const long long from = at.b * a.xb + at.col, up = static_cast<long long>(at.b) * a.N * a.C + at.col;
    for (int n = at.n0 + at.row; n < at.n1; n += U * a.rows) {
        float x[U][V], dy[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int m = min(n + u * a.rows, at.n1 - 1);
            load_piece<T, V>(a.x, from + m * a.xn, x[u]);
            load_piece<T, V>(a.dy, up + static_cast<long long>(m) * a.C, dy[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n + u * a.rows >= at.n1) break;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float v = (x[u][i] - ch.mean[i]) * ch.r[i], dz = dy[u][i] * slope(v * ch.w[i] + ch.bias[i], a.act);
                x[u][i] = ch.r[i] * (dz * ch.w[i] - s0[i] - v * s1[i]);
            }
            store_piece<T, V>(a.dx, up + static_cast<long long>(n + u * a.rows) * a.C, x[u]);
        }
    }
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
    a.blocks = p.blocks;
    a.parts = p.parts;
    a.lanes = p.lanes;
    a.div_N = make_fastdiv(a.N);
    a.div_P = make_fastdiv(a.P);
    const unsigned param_blocks = a.dweight || a.dbias ? static_cast<unsigned>((a.C + 31) / 32) : 0;
    if (p.tokens) {
        a.sums = p.grid;
        if (!back) launch_tokens<T, V, false>(a, p, stream);
        else launch_tokens<T, V, true>(a, p, stream);
        if (back && param_blocks) hipLaunchKernelGGL(norm_params_kernel, dim3(param_blocks), dim3(kT), 0, stream, a);
        return hipGetLastError();
    }
    a.entries = a.groups * p.parts;
    a.sums = a.B * p.slabs;
    const unsigned grid = static_cast<unsigned>(a.B) * p.slabs * p.blocks;
    const size_t groups_lds = static_cast<size_t>(p.parts == 1 ? std::max(1, std::min(a.groups, p.cols * V / a.P)) : 1) * sizeof(float2);
    if (!back) {
        const int each = a.P % V == 0 ? 1 : V;
        hipLaunchKernelGGL((norm_stats_kernel<T, V>), dim3(grid), dim3(kT), static_cast<size_t>(p.rows) * p.cols * each * sizeof(float2), stream, a);
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
