// Differential attention: argument blocks, and the tiles and matrix fragments its kernels share.
//
//   O = P_0 V - lambda P_1 V,   P_m = softmax(scale Q_m K_m^T) over the visible keys,   m = 0, 1
//
// All products run on the 32x32 MFMA, contracted 16 elements at a time. A fragment is one lane's 8 elements of such a
// step: lane l holds row l & 31, elements 8 (l >> 5) .. + 7 (bf16: one 32x32x16 instruction; fp32: eight 32x32x2 ones,
// which take the elements in another order, the same on both sides). A result lane holds column l & 31 and rows
// 8 (r >> 2) + 4 (l >> 5) + (r & 3) for r = 0 .. 15: eight of them, packed, are a fragment of the next product whose
// contraction runs over those rows, in the order 4h .. 4h+3, 8+4h .. 8+4h+3 (h = l >> 5). The other operand of that
// product is read from LDS in the same order (col_frag), so scores never leave their lanes.
#ifndef QTA_DIFF_ATTN_H
#define QTA_DIFF_ATTN_H

#include <algorithm>

#include "bf16_tiles.h"
#include "qta_internal.h"

namespace qta {

struct DiffArgs {
    const void* q;              // [B][Nq][2 heads][d], by strides; head i's maps are 2i and 2i + 1
    const void* k;              // [B][Nk][2 kv_heads][d]
    const void* v;              // [B][Nk][kv_heads][2d]
    const void* lam;            // fp32, or bf16 with lam_bf16
    bool lam_bf16, causal;
    int B, heads, kv_heads, Nq, Nk;
    int R;                      // Nq * (heads / kv_heads) rows of one key head: row r is query r / G of its head r % G
    FastDiv div_G;
    long long qb, qn, qh, kb, kn, kh, vb, vn, vh, lb, ln, lh;   // strides in elements
    const int32_t* lens;        // [B] keys of each batch element, or NULL
    const int32_t* q_pos;       // [B] key position of query 0 (causal), or NULL: Nk - Nq
    float scale;                // of the logits, times log2(e): weights are powers of two
    void* out;                  // [B][Nq][heads][2d]
    // kept for the backward (NULL in inference): P_0 V and P_1 V, fp32 [B][Nq][heads][2][2d] (from the rounded output dQ
    // and dK of short causal sequences are 1.6 times as far off as rounding makes a result, from these 1.45), and log2 of
    // the weights' sums [B][heads][2][Nq] (-inf where a row sees nothing)
    float* maps;
    float* lse;
    // few rows: waves split the keys of a tile instead of rows, and the keys come in `splits` parts (see diff_key_parts),
    // whose results go to part, fp32 [splits][B][kv_heads][2][R][2d], and part_sums, [..][R][2] (maximum, sum)
    bool keys_apart;
    int splits;
    float* part;
    float* part_sums;
};

// How a forward's keys are split. Up to 32 rows of a key head (a token or a few, of all the query heads that share it): the
// waves of a workgroup take halves of each key tile, since half of them would find no rows (16 tokens over caches of 16384
// to 32768 keys, 32 heads over 8, d = 64, bf16: 270 us, by rows 292; 8 x 5 tokens over 4097 keys, 16 heads over 4,
// d = 32, fp32: 22 us, by rows 32). And where the rows do not give every unit a workgroup (fp32, whose products take 16
// times as long: two), the keys come in parts that make four workgroups a unit, none below 256 keys (4800 fp32 tokens,
// 4 heads, d = 32: 510 us whole, 381 in two parts, 327 in four; the long caches: 289 us with two workgroups a unit, 274 with
// four, 280 with eight; the fp32 caches: 31 us in parts of 256 keys, 38 in parts of 128; below 1024 bf16 keys the second
// launch costs more than it gives: 512 keys, 8 heads, d = 64, 12 us a call whole, 16 in two parts). Parts cost a write and a read
// of fp32 results: 3 x 1031 bf16 tokens over 1777, 8 heads, d = 32, which are 408 workgroups, take 31 us, in three
// parts 30 and 14 to join them.
struct DiffParts {
    bool keys_apart;
    int splits;
};
inline DiffParts diff_key_parts(int B, int kv_heads, int Nk, int R, bool bf16_inputs)
{
    const long long groups = static_cast<long long>(B) * kv_heads, cus = device_cu_count();
    DiffParts p{false, 1};
    const long long tiles = groups * ((R + 63) / 64);
    if (tiles >= (bf16_inputs ? cus : 2 * cus) && R > 32) return p;
    p.keys_apart = R <= 32;
    const long long work = groups * ((R + (p.keys_apart ? 31 : 63)) / (p.keys_apart ? 32 : 64));
    const long long want = (4 * cus + work - 1) / work, most = bf16_inputs && Nk < 1024 ? 1 : Nk / 256;
    p.splits = static_cast<int>(most < 1 ? 1 : want < 1 ? 1 : want > most ? most : want);
    if (p.splits > 64) p.splits = 64;
    return p;
}

// The visible range of one batch element: keys [0, len), and for query i of a causal call those up to pos + i.
struct DiffRange {
    int len, pos;
    bool causal;
    __device__ __forceinline__ int limit(int i) const { return causal ? max(0, min(len, pos + i + 1)) : len; }
    // the query that query i is read as: itself, or, where it sees no key and may hold anything, the first that does
    __device__ __forceinline__ int read_as(int i, int Nq) const { return causal ? max(i, min(-pos, Nq - 1)) : i; }
};
__device__ __forceinline__ DiffRange diff_range(const DiffArgs& a, int b)
{
    DiffRange r;
    r.len = a.lens ? min(max(a.lens[b], 0), a.Nk) : a.Nk;
    // (clamped so that pos + i + 1 cannot overflow; nothing changes in what is visible)
    r.pos = a.causal ? (a.q_pos ? min(max(a.q_pos[b], -a.Nq - 1), a.Nk) : a.Nk - a.Nq) : 0;
    r.causal = a.causal;
    return r;
}

__device__ __forceinline__ float diff_lambda(const DiffArgs& a, int b, int i, int h)
{
    const long long at = b * a.lb + i * a.ln + h * a.lh;
    return a.lam_bf16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(a.lam)[at]) : static_cast<const float*>(a.lam)[at];
}

namespace diff {

using tiles::bf16x8_t;
using tiles::lds_byte;
using tiles::lds_ptr;
using tiles::pack2;
using tiles::short4_t;
using tiles::u32x4_t;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Frag;
template <> struct Frag<bf16> {
    bf16x8_t v;
};
template <> struct Frag<float> {
    float v[8];
};

__device__ __forceinline__ f32x16 mma(const Frag<bf16>& a, const Frag<bf16>& b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

// 16 bytes at p as part of a fragment; a fragment of 8 elements in memory.
__device__ __forceinline__ void frag_from(Frag<bf16>& f, const u32x4_t& x, int) { f.v = __builtin_bit_cast(bf16x8_t, x); }
__device__ __forceinline__ void frag_from(Frag<float>& f, const u32x4_t& x, int part)
{
    const f32x4 y = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[4 * part + i] = y[i];
}
template <typename T>
__device__ __forceinline__ Frag<T> global_frag(const void* base, long long elem)
{
    constexpr int parts = sizeof(T) / 2;
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(static_cast<const unsigned char*>(base) + elem * static_cast<long long>(sizeof(T)));
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < parts; ++i) frag_from(f, p[i], i);
    return f;
}

// Result rows 8s .. 8s + 7 (in the order above) as a fragment. bf16: rounded to nearest, 2^-8 of each value at
// most, once, as the matrix product asks; sums of weights are taken from the fp32 values.
template <typename T>
__device__ __forceinline__ Frag<T> pack_frag(const float* x)
{
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
        u32x4_t w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2(x[2 * i], x[2 * i + 1]);
        f.v = __builtin_bit_cast(bf16x8_t, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = x[i];
    }
    return f;
}

// LDS at a byte address.
template <typename V>
__device__ __forceinline__ lds_ptr<V> lds_at(uint32_t at)
{
    return (lds_ptr<V>)static_cast<uintptr_t>(at);
}
__device__ __forceinline__ uint32_t lds_address(lds_byte* p) { return static_cast<uint32_t>((uintptr_t)p); }

// A tile of rows of W elements in LDS, in 16-byte chunks: chunk c of row r lies at place c ^ swz(r) of its row. The
// swizzle spreads both ways of reading over all banks: 16 lanes on one chunk of 16 rows (row_frag), and for bf16 four
// rows times 64 bytes (col_frag, transposed by the read). fp32 column reads meet two to a bank where a row is 128 bytes,
// which an fp32 product (64 cycles for 2 of the 16 elements) hides.
template <typename T, int W>
struct Tile {
    static constexpr int kRow = W * static_cast<int>(sizeof(T));
    static constexpr int kChunks = kRow / 16;              // 4, 8, 16 or 32
    static constexpr int bytes(int rows) { return rows * kRow; }

    // (the exclusive or of the swizzles of two rows whose bits do not overlap is that of their sum)
    __device__ static __forceinline__ constexpr int swz(int r)
    {
        if constexpr (kChunks == 4) return (r >> 2) & 3;
        else if constexpr (kChunks == 8) return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1 | ((r >> 3) & 1);
        else if constexpr (sizeof(T) == 2) return (r & 3) << 2 | ((r >> 2) & 3);
        else return ((r >> 2) & 1) << 3 | (r & 3) << 1 | ((r >> 3) & 1);
    }

    // Brings `rows` rows in (a multiple of 64 / kChunks), each wave its share, 1 KB an instruction straight to LDS:
    // `off(r)` is the byte offset of row r in `map`.
    template <typename Off>
    __device__ static __forceinline__ void stage(lds_byte* tile, __amdgpu_buffer_rsrc_t map, int rows, int wave, int waves,
                                                 int lane, Off off)
    {
        constexpr int per = 64 / kChunks;                  // rows an instruction
        static_assert(kChunks <= 32, "rows of at most 512 bytes");
#pragma unroll
        for (int r0 = 0; r0 < rows; r0 += per * waves) {
            const int first = r0 + wave * per;
            if (first >= rows) break;
            const int r = first + lane / kChunks;
            tiles::load_lds16(map, off(r) + static_cast<uint32_t>(((lane % kChunks) ^ swz(r)) * 16), 0, tile + first * kRow);
        }
    }

    // Where a lane's reads start in a tile: row lane & 31 for row fragments, and for column fragments the lane's part of
    // rows 0 .. 15. A step, a column tile or eight rows more flip bits of these (the swizzle's bits lie above the lane's),
    // so a read costs one exclusive or and everything else is an immediate.
    __device__ static __forceinline__ uint32_t row_base(int lane)
    {
        constexpr int parts = sizeof(T) / 2;
        const int r = lane & 31;
        return static_cast<uint32_t>(r * kRow + (((lane >> 5) * parts) ^ swz(r)) * 16);
    }
    __device__ static __forceinline__ uint32_t col_base(int lane)
    {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 rows x 32 bytes, 8 bytes each, and receive one column of the four rows each
            const int i = lane & 15, r = 4 * h + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i >> 1) & 1);
            return static_cast<uint32_t>(r * kRow + (c ^ swz(r)) * 16 + (i & 1) * 8);
        } else {
            const int col = lane & 31;
            return static_cast<uint32_t>(4 * h * kRow + ((col >> 2) ^ swz(4 * h)) * 16 + (col & 3) * 4);
        }
    }

    // Row r0 + (lane & 31), elements 16 step + 8 (lane >> 5) .. + 7, of the tile at `tile`; r0 a multiple of 32.
    __device__ static __forceinline__ Frag<T> row_frag(uint32_t base, uint32_t tile, int r0, int step)
    {
        constexpr int parts = sizeof(T) / 2;
        Frag<T> f;
#pragma unroll
        for (int i = 0; i < parts; ++i) {
            const u32x4_t x = *lds_at<u32x4_t>((base ^ static_cast<uint32_t>((2 * step * parts + i) * 16)) + (tile + r0 * kRow));
            frag_from(f, x, i);
        }
        return f;
    }

    // Column 32 ct + (lane & 31) of rows r0 + 4h .. + 3 and r0 + 8 + 4h .. + 3 (h = lane >> 5), r0 a multiple of 16.
    __device__ static __forceinline__ Frag<T> col_frag(uint32_t base, uint32_t tile, int r0, int ct)
    {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            short4_t x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t flip = static_cast<uint32_t>((4 * ct ^ swz(8 * u)) * 16);
                x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<short4_t>((base ^ flip) + (tile + (r0 + 8 * u) * kRow)));
            }
            f.v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = 8 * (j >> 2) + (j & 3);
                f.v[j] = *lds_at<float>((base ^ static_cast<uint32_t>((8 * ct ^ swz(r)) * 16)) + (tile + (r0 + r) * kRow));
            }
        }
        return f;
    }
};

// Stands in a branch that few tiles take, which the compiler would otherwise turn into selects that all of them take.
__device__ __forceinline__ void branch_here() { asm volatile(""); }

// Keeps a lane's base from being known across iterations: the compiler would otherwise hold every variant of it in a
// register of its own (32 of them in the key pass).
__device__ __forceinline__ void opaque(uint32_t& x) { asm("" : "+v"(x)); }

// Row of result register r in a lane's half h.
__device__ __forceinline__ constexpr int acc_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// Four consecutive elements at p (16-byte aligned for fp32, 8 for bf16).
template <typename T>
__device__ __forceinline__ void store4(void* base, long long elem, float a, float b, float c, float d)
{
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + elem) = make_uint2(pack2(a, b), pack2(c, d));
    } else {
        *reinterpret_cast<float4*>(static_cast<float*>(base) + elem) = make_float4(a, b, c, d);
    }
}

__device__ __forceinline__ const unsigned char* byte_at(const void* p, long long elem, int size)
{
    return static_cast<const unsigned char*>(p) + elem * size;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float other_half(float x) { return xchg_f32<32>(x); }

}  // namespace diff

// Backward: the argument block, and what each pass writes.
struct DiffBwdArgs {
    DiffArgs f;                 // maps and lse are the forward's (read)
    const void* dout;           // [B][Nq][heads][2d] contiguous
    // by rows of one key head, for the key pass: [B][kv_heads][kDiffStats][Rpad] fp32. With s the logits' scale, S the sign
    // of lambda: -lse_0 / s, -(lse_1 - log2 |lambda|) / s (fp32 inputs: both without the division), -t_0, -S (t_0 - t_1), -S
    float* stats;
    int Rpad;                   // R rounded up to kDiffRowPad; rows behind R are zero
    void* dq;                   // [B][Nq][2 heads][d]
    void* dk;                   // [B][Nk][2 kv_heads][d]
    void* dv;                   // [B][Nk][kv_heads][2d]
    void* dlam;                 // lambda's type: [B][Nq][heads], or [heads] with lam_heads
    bool lam_heads;
    float* dlam_rows;           // fp32 [heads][B * Nq] with lam_heads
    float grad_scale;           // scale of the logits
    // the key pass in `splits` parts of the rows: fp32 [splits][B][Nk][kv_heads][4d] sums of dK_0, dK_1 and dV (splits > 1)
    int splits;
    float* part;
    int key_groups;             // workgroups of the key pass that have keys; set by the launcher
    // the query pass in `q_splits` parts of the keys: fp32 [q_splits][B][kv_heads][R][2][d] sums of dQ_0 and dQ_1, and
    // [..][R] those of P_1 (D - t_1), the first part's plus t_1 (q_splits > 1)
    int q_splits;
    float* q_part;
    float* q_miss;
};
constexpr float kDiffLn2 = 0.693147180559945f;
constexpr int kDiffStats = 5;
constexpr int kDiffRowPad = 64;
constexpr int kDiffKeys = 128;  // keys of a workgroup of the key pass

// Parts of the key pass's rows. One key head's keys in tiles of 128 may be few workgroups, and under a causal mask the
// first tile meets all rows and the last only its own; parts cost a write and a read of fp32 sums. Two workgroups run on a
// unit: as many parts as fill the units twice where work is even and four times where it is causal, no part below
// 4 tiles of 32 rows. (2 x 4096 keys, 16 heads over 4, d = 64, bf16, causal: in 2 parts 472 us and 14 to join them, in 4
// parts 357 and 23, in 6 parts 354 and 33.) Past eight parts the sums weigh more: half as many workgroups and no part below
// 8 tiles. (A training step, bf16, d = 64, 8 heads over 1: 7591 queries of 232 keys 579 us in 8 parts, 175 in 128 and 184 in
// 64; 2048 causal tokens 240 in 8, 178 in 32, 186 in 64.)
constexpr int kDiffEvenParts = 8;
inline int diff_key_splits(int B, int kv_heads, int Nk, int R, bool causal)
{
    const long long groups = static_cast<long long>(B) * kv_heads * ((Nk + kDiffKeys - 1) / kDiffKeys);
    const long long want = static_cast<long long>(device_cu_count()) * (causal ? 4 : 2);
    long long s = std::min<long long>((want + groups - 1) / groups, R / 128);
    if (s > kDiffEvenParts)
        s = std::max<long long>(kDiffEvenParts, std::min<long long>((want / 2 + groups - 1) / groups, R / 256));
    return static_cast<int>(std::max(s, 1LL));
}

// Parts of the query pass's keys: enough to give every unit a workgroup, none below 256 keys, at most 64 (2 x 997 causal
// tokens, 8 heads, d = 32, fp32: 103 us whole, 53 in two parts, 60 in three; a training step of 100 queries, 4 heads over 1,
// and 16000 keys, d = 32, fp32: 243 us with at most 16 parts, 177 with 62).
inline int diff_query_splits(int B, int kv_heads, int Nk, int R)
{
    const long long groups = static_cast<long long>(B) * kv_heads * ((R + 127) / 128);
    const long long s = std::min<long long>((device_cu_count() + groups - 1) / groups, Nk / 256);
    return static_cast<int>(std::clamp(s, 1LL, 64LL));
}

// Workgroups of the launches, as the launchers make them and the entry points check them beforehand: HIP takes fewer than
// 2^32 threads a launch, which is 2^24 workgroups.
constexpr int kDiffThreads = 256;
constexpr long long kDiffMaxBlocks = (1LL << 32) / kDiffThreads - 1;
inline long long diff_fwd_blocks(long long groups, long long R, const DiffParts& p)
{
    const int rows = p.keys_apart ? 32 : 64;
    return (R + rows - 1) / rows * groups * p.splits;
}
inline long long diff_join_blocks(long long groups, long long R)       // a wave a row
{
    return (groups * R + kDiffThreads / kWave - 1) / (kDiffThreads / kWave);
}
inline long long diff_dq_blocks(long long groups, long long R, int q_splits) { return (R + 127) / 128 * groups * q_splits; }
inline long long diff_dq_join_blocks(long long groups, long long R, int d)
{
    return (groups * R * (d / 2) + kDiffThreads - 1) / kDiffThreads;
}
inline long long diff_dkv_blocks(long long groups, long long Nk, int splits) { return (Nk + kDiffKeys - 1) / kDiffKeys * groups * splits; }
inline int diff_dkv_slices(int splits) { return splits > kDiffEvenParts ? 8 : 1; }             // many parts are of few keys
inline long long diff_dkv_join_blocks(long long groups, long long Nk, int d, int splits)
{
    return (groups * Nk * d * diff_dkv_slices(splits) + kDiffThreads - 1) / kDiffThreads;
}

hipError_t launch_diff_attn(const DiffArgs& a, int d, bool use_bf16, hipStream_t stream);
hipError_t launch_diff_bwd(const DiffBwdArgs& a, int d, bool use_bf16, hipStream_t stream);

// Rotary positions of one or two tensors.
struct RotaryTensor {
    const void* x;
    void* y;
    int heads;
    long long xb, xn, xh, yb, yn, yh;
};
struct RotaryArgs {
    RotaryTensor t[2];
    int B, N, d, rot, axes, width;
    bool interleaved, inverse;
    const double* freqs;        // [rot / 2] radians a position
    const int32_t* pos;         // [B][N][axes], stride pos_b elements between batch elements; or NULL
    long long pos_b;
    int start;
    float scale;
    FastDiv div_N, div_W, div_pairs, div_items, div_heads;      // set by the launcher
    int items, tokens;          // items of a head, tokens of a workgroup; set by the launcher
    long long first;            // token of the launch's first workgroup; set by the launcher
};
hipError_t launch_rotary(const RotaryArgs& a, bool use_bf16, hipStream_t stream);

}  // namespace qta

#endif
