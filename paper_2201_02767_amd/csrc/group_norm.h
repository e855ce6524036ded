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
    int cols, rows, slabs, slab, blocks, parts, entries;
    unsigned own;               // workgroups of the launch that have tokens
    int lanes, sums;            // (per token) lanes of a group; workgroups' sums in part
    int rows_lanes;             // lanes that share the rows of a channel
    float* group_part;
    FastDiv div_N, div_P, div_slabs, div_rows, div_entry;
};

// Maps take two launches that each go over them (bound by memory: 8 maps of 200 x 336 x 256 bf16, 275 MB each, SiLU: 46 us to read x, 105 to
// read it and write y, 100 to read x and dy, 155 to read them and write dx, 5.2 to 6.0 TB/s, where a large copy makes 5.1). The second
// goes through every slab from its end, where the memory's cache still holds what the first read last, and stores go past the caches (with
// ordinary stores, whose lines the next kernel's reads push out, and upwards: 71, 95, 150 and 164 us).
// Batch elements one after the other, which would fit the caches, fill the card too badly: 467 us for these 407.
//
// A workgroup of kNormThreads threads takes a block of `cols` vector columns, `rows` tokens at a time, of one slab of the tokens of
// a batch element. A thread's channels stay the same, and its sums over tokens stay in registers. Blocks hold whole groups, or
// where a group is wider than a workgroup, a part of one (`parts` a group).
constexpr int kNormThreads = 1024;

struct NormPlan {
    bool tokens;                // every token by itself: its groups in registers, or `wide`, a group a workgroup
    bool wide;
    int V;                      // elements of an access
    int cols, rows, slabs, slab, blocks, parts;      // slab: its tokens
    int lanes, pieces, grid;    // per token: lanes of a group, accesses of a lane, workgroups
    // of `part`: in the backward [sums][C] (sum dz n, sum dz), sums = B * slabs, or per token `grid`; then but per token
    // [B][slabs][groups * parts] (forward: mean, sum of squared distances; backward: sum dn n, sum dn)
    size_t channel_floats;
    size_t bytes;
};

constexpr int kNormMaxPieces = 4;

// `align`: elements that everything about x, y, dy and dx (addresses, strides) is a multiple of, a power of two up to 16 bytes.
inline NormPlan norm_plan(int B, int N, int C, int groups, bool per_token, bool bf16_inputs, int align, bool back)
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
        // four workgroups a unit, each with its own sums for the weights (16384 tokens of 16 x 128, bf16: forward and backward 29 and 43 us,
        // 4.7 TB/s, and 6 for the sums; two a unit take 1.2 times as long and 4, eight as long forward, 1.2 times as long backward, and 11)
        const long long tokens = (static_cast<long long>(B) * N + p.rows - 1) / p.rows;
        p.grid = static_cast<int>(std::min<long long>(tokens, std::max(1LL, 4LL * device_cu_count() / p.blocks)));
        p.bytes = back ? static_cast<size_t>(p.grid) * C * 2 * sizeof(float) : 0;
        return p;
    }
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
    // one workgroup a unit: half as many threads in twice as many, or two a unit, read more of the slabs' sums in all (2 x 19200 tokens
    // of 256 channels, bf16: the second launch takes 11.8 us; when it took 16 they took 22 and 30). Where batch elements and blocks leave slabs uneven over
    // the units, four times as many.
    const long long want = device_cu_count(), wide = static_cast<long long>(B) * p.blocks;
    const long long many = want / wide >= 8 ? want / wide : (4 * want + wide - 1) / wide;
    const long long slabs = std::max(1LL, std::min<long long>(many, (N + 4 * p.rows - 1) / (4 * p.rows)));
    p.slab = static_cast<int>((N + slabs - 1) / slabs);
    p.slabs = (N + p.slab - 1) / p.slab;
    const size_t sums = static_cast<size_t>(B) * p.slabs;
    p.channel_floats = back ? sums * C * 2 : 0;
    p.bytes = (p.channel_floats + sums * groups * p.parts * 2) * sizeof(float);
    return p;
}

hipError_t launch_norm_forward(const NormArgs& a, const NormPlan& p, bool use_bf16, hipStream_t stream);
hipError_t launch_norm_backward(const NormArgs& a, const NormPlan& p, bool use_bf16, hipStream_t stream);

}  // namespace qta

#endif
