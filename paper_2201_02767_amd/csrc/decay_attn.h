// Linear attention with a decay: argument blocks and the rules by which its work is divided.
//
//   S_t = exp(g) S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
//
// Over a chunk of C tokens behind a state S (i, j = 0 .. C-1 within the chunk):
//   o_i = f exp(g (i + 1 - e)) S^T q_i + scale sum over j <= i of exp(g (i - j)) (q_i . k_j) v_j
//   S  <- exp(g C) S + u sum over j of exp(g (C - 1 - j + e)) k_j v_j^T
// with e = 0, f = scale, u = 1 in the forward. The gradients are the same sums. With R the loss's gradient with respect to the state,
//   dq_t = scale S_t do_t:                  the forward with (do, v, k) for (q, k, v) and S transposed;
//   dv_s = R_s^T k_s, dk_s = R_s v_s,       R_s = exp(g) R_{s+1} + scale q_s do_s^T: with time running back, (k, q, do) and
//                                           (v, do, q), and e = 1, f = 1, u = scale, since R starts as the gradient of the last state.
// So one kernel serves all four; a role says what is read as q, k and v, and which way.
#ifndef QTA_DECAY_ATTN_H
#define QTA_DECAY_ATTN_H

#include <algorithm>

#include "diff_attn.h"

namespace qta {

struct DecayRole {
    const void *q, *k, *v;                                      // [B][N][heads][.] by strides in elements
    long long qb, qn, qh, kb, kn, kh, vb, vn, vh;
    void* out;                  // [B][N][heads][DV] contiguous
    const float* state;         // before the first token, or (with several segments) before each segment; NULL: zeros
    int s_row, s_col;           // its strides (a transposed state has s_row = 1)
    float* last;                // the state behind the last token, laid out like `state`, from calls of one segment; or NULL
    bool back;                  // time runs back: e = 1
    float f, u;                 // see above
};

struct DecayArgs {
    DecayRole role[3];
    int roles, B, heads, N;
    int segs, seg;              // a (batch, head)'s tokens in `segs` segments of `seg` tokens
    FastDiv div_segs, div_heads;
    const float* log_decay;
    const int32_t* lens;
    float scale;
    float* part;                // fp32 [roles][B][heads][segs][DK][DV]: what each segment adds to the state, then the states before them
};

// The scan over segments: part[r] becomes the states before each segment, and last[r] the one behind the last.
struct DecayScanArgs {
    float* part;
    const float* state[2];      // before the first token, NULL: zeros
    float* last[2];             // may be state itself; NULL: not asked for
    int B, heads, N, segs, seg, cells;      // cells: dk * dv
    const float* log_decay;
    const int32_t* lens;
};

struct DecayStepArgs {
    const void *q, *k, *v;
    long long qb, qn, qh, kb, kn, kh, vb, vn, vh;
    void* out;
    const float* state;         // NULL: zeros
    float* last;                // NULL: not asked for
    int B, heads, N;
    FastDiv div_heads;
    const float* log_decay;
    const int32_t* lens;
    float scale;
};

// Calls of up to this many tokens go token by token through states that stay in registers.
constexpr int kDecayStepTokens = 16;
// Workgroups that share the columns of a head's state in them, 64 each.
constexpr int decay_step_slices(int dv) { return dv < 64 ? 1 : dv / 64; }

// Tokens of a chunk: a tile of the products.
constexpr int kDecayChunk = 32;
constexpr int kDecayTables = 4096 + 2 * kDecayChunk * 4;            // bytes of the weights behind the chunks in LDS
// Chunks in LDS at a time: as many as leave room for three workgroups of the largest kind (a unit has 160 KB), at most four. (The loads
// of two are enough: with two, three and four chunks prompts of 65536 tokens take the same 200 us.)
constexpr int decay_depth(int bytes) { return 4 * bytes <= (48 << 10) ? 4 : 3 * bytes <= (48 << 10) ? 3 : 2; }

// Waves a SIMD that the kernels' registers are held to: as many as they fit without going to memory inside the chunks' loop, or nearly so (2 x
// 8192 bf16 tokens, 16 heads of 128/64: 64 us with two, 81 with three and 18 registers in memory; 2 x 4096 fp32 tokens, 16 heads of
// 128/32: 93 us with one, 131 with two and 163 in memory; of 128/64 142 with two and 18, 144 with one).
constexpr int decay_waves(bool bf16_inputs, int dk, int dv)
{
    if (bf16_inputs) return dk == 128 && dv < 128 ? 2 : 3;
    return dk == 32 ? 3 : dk == 128 && dv == 32 ? 1 : 2;
}

// Segments of a call: enough for two workgroups of four waves a unit, or as many waves in smaller ones (2 x 8192 tokens, 16 heads of 128,
// bf16, forward and backward: states 57 + 57, scans 12 + 12, results 88 + 230 us; with four a unit 60 + 60, 23 + 23 and 88 + 239: the
// states' bytes), none below two chunks, or one in fp32, whose products take 16 times as long (2 x 997 tokens, 8 heads of 32, a step's five
// launches 53 us with two, 44 with one; 3 x 1031 bf16 tokens, 8 heads of 32/64: as long with two as with one, 1.4 times with eight).
struct DecaySegments {
    int segs, seg;
};
// `dv`: the width that makes the workgroups' waves; in a backward, whose launches have either width, the smaller (a backward of 2 x 4096
// fp32 tokens, 16 heads of 128/32: 298 us by the larger, 245 by the smaller).
inline DecaySegments decay_segments(int B, int heads, int N, int dv, int roles, bool bf16_inputs)
{
    const long long rows = static_cast<long long>(B) * heads * roles, want = 2LL * device_cu_count() * 128 / dv;
    const long long most = std::max(1, N / ((bf16_inputs ? 2 : 1) * kDecayChunk));
    const long long segs = std::max(1LL, std::min(most, (want + rows - 1) / rows));
    const int seg = static_cast<int>(((N + segs - 1) / segs + kDecayChunk - 1) / kDecayChunk * kDecayChunk);
    return {(N + seg - 1) / seg, seg};
}

constexpr long long kDecayMaxBlocks = (1LL << 32) / 256 - 1;

hipError_t launch_decay_step(const DecayStepArgs& a, int dk, int dv, bool use_bf16, hipStream_t stream);
// What the segments add to the states (roles' k and v).
hipError_t launch_decay_states(const DecayArgs& a, int dk, int dv, bool use_bf16, hipStream_t stream);
hipError_t launch_decay_scan(const DecayScanArgs& a, int roles, hipStream_t stream);
// The results of a's roles; dk, dv are the sizes as the roles read them.
hipError_t launch_decay_chunks(const DecayArgs& a, int dk, int dv, bool use_bf16, hipStream_t stream);

}  // namespace qta

#endif
