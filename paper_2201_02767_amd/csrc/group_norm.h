// Group norm with an activation, channels last: argument block and the rules by which its work is divided.
//
//   n = (x - mean) r,  r = 1 / sqrt(var + eps),  y = act(w n + b)
//   dz = dy act'(w n + b),  dn = w dz,  dx = r (dn - mean(dn) - n mean(dn n)),  dw = sum dz n,  db = sum dz
#ifndef QTA_GROUP_NORM_H
#define QTA_GROUP_NORM_H

#include <algorithm>

#include "qta_internal.h"

namespace qta {

struct NormArgs {
    const void* x;
    const void* weight;         // NULL: 1
    const void* bias;           // NULL: 0
    bool param_bf16;
    int B, N, C, groups, P;     // P: channels of a group
    long long xb, xn;           // strides of x in elements
    int act;
    float eps;
    void* y;
    float* stats;               // [B][groups][2] mean and r, or NULL
    // backward
    const void* dy;             // contiguous
    void* dx;
    void* dweight;              // NULL: not asked for
    void* dbias;
    float* part;                // see NormPlan
    // set by the launchers from the plan
    int cols, rows, slabs, blocks, parts, entries;
    int lanes, sums;            // (per token) lanes of a group; workgroups' sums in part
    FastDiv div_N, div_P;
};

// Maps: a workgroup of kNormThreads threads takes a block of `cols` vector columns, `rows` tokens at a time, of one slab of the tokens of
// a batch element. A thread's channels stay the same, and its sums over tokens stay in registers. Blocks hold whole groups, or
// where a group is wider than a workgroup, a part of one (`parts` a group).
constexpr int kNormThreads = 512;

struct NormPlan {
    bool tokens;                // every token by itself: its groups in registers, or `wide`, a group a workgroup
    bool wide;
    int V;                      // elements of an access
    int cols, rows, slabs, blocks, parts;
    int lanes, pieces, grid;    // per token: lanes of a group, accesses of a lane, workgroups
    // bytes of `part`: forward [B][slabs][groups * parts] (mean, sum of squared distances); backward [sums][C] (sum dz n, sum dz),
    // sums = B * slabs, or per token `grid`
    size_t fwd_bytes, bwd_bytes;
};

constexpr int kNormMaxPieces = 4;

inline int norm_gcd(int a, int b) { return b ? norm_gcd(b, a % b) : a; }

// `align`: elements that everything about x, y, dy and dx (addresses, strides) is a multiple of, a power of two up to 16 bytes.
inline NormPlan norm_plan(int B, int N, int C, int groups, bool per_token, bool bf16_inputs, int align)
{
    NormPlan p{};
    const int P = C / groups;
    int V = align;
    while (P % V != 0) V /= 2;
    // a group's lanes lie in one wave and hold it whole
    int lanes = 1;
    while (lanes < 64 && lanes * V < P) lanes *= 2;
    int pieces = 1;
    while (pieces * lanes * V < P) pieces *= 2;
    if (per_token) {
        p.tokens = true;
        p.V = V;
        p.lanes = lanes;
        p.pieces = pieces;
        const int slots = 256 / lanes;
        p.wide = pieces > kNormMaxPieces;
        p.cols = p.wide ? 1 : std::min(groups, slots);              // groups of a workgroup
        p.rows = p.wide ? 1 : slots / p.cols;                       // tokens of a workgroup at a time
        p.blocks = (groups + p.cols - 1) / p.cols;
        const long long tokens = (static_cast<long long>(B) * N + p.rows - 1) / p.rows;
        p.grid = static_cast<int>(std::min<long long>(tokens, std::max(1LL, 4LL * device_cu_count() / p.blocks)));
        p.bwd_bytes = static_cast<size_t>(p.grid) * C * 2 * sizeof(float);
        return p;
    }
    const long long units = B;
    const int tokens = N;
    p.parts = 1;
    p.V = align;
    while (C % p.V != 0) p.V /= 2;
    if (C <= kNormThreads * p.V) {
        p.cols = C / p.V;
        p.blocks = 1;
    } else {
        p.V = V;
        if (P <= kNormThreads * V) {
            const int g = kNormThreads * V / P;
            p.cols = g * P / V;
            p.blocks = (groups + g - 1) / g;
        } else {
            const int pieces_all = P / V;
            p.parts = (pieces_all + kNormThreads - 1) / kNormThreads;
            p.cols = (pieces_all + p.parts - 1) / p.parts;
            p.parts = (pieces_all + p.cols - 1) / p.cols;
            p.blocks = groups * p.parts;
        }
    }
    p.rows = kNormThreads / p.cols;
    const long long want = 2LL * device_cu_count(), wide = units * p.blocks;
    p.slabs = static_cast<int>(std::max(1LL, std::min<long long>((want + wide - 1) / wide, (tokens + 4 * p.rows - 1) / (4 * p.rows))));
    p.fwd_bytes = static_cast<size_t>(units) * p.slabs * groups * p.parts * 2 * sizeof(float);
    p.bwd_bytes = static_cast<size_t>(units) * p.slabs * C * 2 * sizeof(float);
    return p;
}

hipError_t launch_norm_forward(const NormArgs& a, const NormPlan& p, bool use_bf16, hipStream_t stream);
hipError_t launch_norm_backward(const NormArgs& a, const NormPlan& p, bool use_bf16, hipStream_t stream);

}  // namespace qta

#endif
