// Attention, backward: the kernels (fmt_attention.h has the mathematics and the layouts), compiled per head size in
// fmt_attention_bwd_64.hip and fmt_attention_bwd_128.hip.
//
// P is made again from Q, K and lse.  Two kernels: one takes rows and adds up dQ over keys, the other takes keys and adds up dK and dV over
// rows, so that every sum is in one workgroup's accumulators, in a fixed order, at the price of S and dP twice (7 products instead of 5).
//
// Measured: 4 x 1024 tokens, 16 heads of 64, window 256 and 4 sinks, bfloat16: 65 us for the 9.5 GFLOP of five products over the pairs that are
// seen (146 TFLOP/s), beside 16 for the packing and 6 for the sinks' parts.  Bound by the vector units and by waiting (the matrix cores are busy for 19 % of
// the time, LDS for 20 %; waves wait for 43 % of theirs): registers leave two waves to a SIMD, and between two products
// lie an exponential, the factors of P and dS and the conversions of every score.
#pragma once

#include "fmt_attention.h"

namespace fmt {

struct AttnBwd {
    AttnShape s;
    AttnView q, k, v, o, go, dq, dk, dv;
    const float *lse;
    float *info;              // what the products need of a row, [4][batch][kv_heads][row_tiles * 128]: kInfo*
    uint16_t *qh, *gh;        // fp16 operands: [batch][kv_heads][row_tiles * 128][32 DT] Q and dO, zero past the last row and column,
    uint16_t *kh, *vh;        // [batch][kv_heads][key_tiles * 128][32 DT] K and V, zero past the sequence's length
    uint32_t *highs;          // what is to know of each 32 rows of Q and dO, then of each 32 keys of K, then of V (join)
    float *part;              // [2][parts][batch][part_keys][kv_heads][dim] of dK, dV
    float up;                 // what the fp16 operands are multiplied by
    bool check;               // whether that has a limit
    float limit;              // of Q and K
    float whole;              // what fp16 operands hold with all of their bits, as they are held
    bool codes, gcodes;       // how q, k and v, and o and go, are stored
    int32_t parts;            // parts of the rows that each of the first part_tiles tiles of keys adds up
    int32_t part_keys;        // their keys
    uint32_t part_tiles, key_tiles, row_tiles, key_blocks, row_blocks;
    int32_t result;
    ElemFormat f;
};

// lse in base 2, and +infinity where a row sees nothing, which makes its P zero; delta; the power of two that brings the row of
// dO to [2^11, 2^12), as its exponent (kNoRow: the row is zero), and delta times that.
enum : int { kInfoLse2 = 0, kInfoDelta = 1, kInfoGrow = 2, kInfoScaledDelta = 3 };
constexpr float kNoRow = 1024.0f;

constexpr int kRowTile = 128, kKeyTile = 64, kKvKeys = 128, kKvRows = 32, kPackRows = 32;

__device__ __forceinline__ int64_t info_rows(const AttnBwd &a) { return static_cast<int64_t>(a.s.batch) * a.s.kv_heads * a.row_tiles * kRowTile; }

// Row r of the heads that share a kv head: its token and its head among them.
struct RowAt {
    int t, g;
};
__device__ __forceinline__ RowAt row_at(int row, int group)
{
    if (group == 1) return RowAt{row, 0};
    const int t = static_cast<int>(static_cast<uint32_t>(row) / static_cast<uint32_t>(group));
    return RowAt{t, row - t * group};
}

// The kernels of one head size (DT blocks of 32 columns); half: with fp16 operands, in one or two pieces of P and dS.
template <int DT>
void run_attention_bwd(const AttnBwd &a, bool half, bool two, dim3 blocks, hipStream_t stream);

namespace {

// Rows whose dQ a workgroup adds up over keys.  The later ones of a causal mask see more keys: they go first.
struct RowBlock {
    int b, kh, row0, row, t, head, pos, rows;
    bool live;
    int64_t i0, i1, info;
    AttnSeq seq;
};
__device__ __forceinline__ RowBlock row_block(const AttnBwd &a, uint32_t id)
{
    const AttnShape &s = a.s;
    RowBlock r;
    const uint32_t tile = id % a.row_tiles, rest = id / a.row_tiles;
    r.kh = static_cast<int>(rest % s.kv_heads);
    r.b = static_cast<int>(rest / s.kv_heads);
    r.row0 = static_cast<int>(s.causal ? a.row_tiles - 1 - tile : tile) * kRowTile;
    r.rows = s.q_len * s.group;
    r.row = r.row0 + static_cast<int>(threadIdx.x >> 6) * 32 + static_cast<int>(threadIdx.x & 31);
    const RowAt at = row_at(r.row, s.group);
    r.t = at.t;
    r.head = r.kh * s.group + at.g;
    r.live = r.row < r.rows;
    r.seq = attn_seq(s, r.b);
    r.pos = r.seq.first + r.t;
    r.i0 = static_cast<int64_t>(r.seq.first) + r.row0 / s.group;
    r.i1 = static_cast<int64_t>(r.seq.first) + (min(r.row0 + kRowTile, r.rows) - 1) / s.group;
    r.info = (static_cast<int64_t>(r.b) * s.kv_heads + r.kh) * a.row_tiles * kRowTile + r.row;
    return r;
}

template <int DT>
__device__ __forceinline__ void store_dq(const AttnBwd &a, const RowBlock &r, const f32x16 (&dq)[DT], float scale)
{
    if (!r.live) return;
    const int half = (threadIdx.x & 63) >> 5;
    store_row<DT>(const_cast<void *>(a.dq.p), r.b * a.dq.sb + r.t * a.dq.st + r.head * a.dq.sh, half, a.s.dim, dq, scale, a.result, a.f);
}

template <int DT>
struct DqShared {
    AttnTile<kPieces, DT, kKeyTile> ks, vs;
};

template <int DT>
__device__ __forceinline__ void dq_pieces(const AttnBwd &a, uint32_t id, DqShared<DT> &sh)
{
    constexpr int NQ = kPieces, NP = kProbPieces;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const RowBlock r = row_block(a, id);
    const int b = r.b, kh = r.kh;

    u32x4 q[2 * DT][NQ], go[2 * DT][NQ];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half, count = r.live ? min(s.dim - col, 8) : 0;
        float v[8], g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = g[j] = 0.0f;
        if (count > 0) {
            load8_any(a.q.p, b * a.q.sb + r.t * a.q.st + r.head * a.q.sh + col, count, v, a.codes, a.f);
            load8_any(a.go.p, b * a.go.sb + r.t * a.go.st + r.head * a.go.sh + col, count, g, a.gcodes, a.f);
        }
        bf16_pieces<NQ>(v, q[kk]);
        bf16_pieces<NQ>(g, go[kk]);
    }
    const int64_t all_rows = info_rows(a);
    const float lse2 = r.live ? a.info[kInfoLse2 * all_rows + r.info] : INFINITY, delta = r.live ? a.info[kInfoDelta * all_rows + r.info] : 0.0f;

    f32x16 dq[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.0f;
    const int64_t kbase = b * a.k.sb + kh * a.k.sh, vbase = b * a.v.sb + kh * a.v.sh;
    const AttnTiles tiles = attn_tiles(s, r.seq.length, r.i0, r.i1, kKeyTile);
    for (int n = 0; n < tiles.count(); ++n) {
        const int k0 = tiles.at(n) * kKeyTile;
        __syncthreads();
        load_tokens<NQ, DT, kKeyTile>(sh.ks, a.k.p, kbase, a.k.st, k0, r.seq.length, s.dim, a.codes, a.f);
        load_tokens<NQ, DT, kKeyTile>(sh.vs, a.v.p, vbase, a.v.st, k0, r.seq.length, s.dim, a.codes, a.f);
        __syncthreads();
        const bool all = attn_sees_all(s, r.seq.length, r.i0, r.i1, k0, k0 + kKeyTile);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                u32x4 f[NQ];
                read_rows(sh.ks, 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                x = mfma_pieces<NQ, NQ>(f, q[kk], x);
                read_rows(sh.vs, 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                dp = mfma_pieces<NQ, NQ>(f, go[kk], dp);
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float ds[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = 8 * kb + j;
                    float y = x[i] * s.scale2;
                    if (!all && !attn_sees(s, r.seq.length, r.pos, k0 + 32 * kt + 8 * (i / 4) + 4 * half + (i & 3))) y = -INFINITY;
                    const float p = exp2_fast(y - lse2);
                    ds[j] = p == 0.0f ? 0.0f : p * (dp[i] - delta);
                }
                u32x4 pp[NP];
                bf16_pieces<NP>(ds, pp);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[NQ];
                    read_columns(sh.ks, 32 * kt + 16 * kb, 32 * d, lane, f);
                    dq[d] = mfma_pieces<NQ, NP>(f, pp, dq[d]);
                }
            }
        }
    }
    store_dq<DT>(a, r, dq, s.scale);
}

// Rows [row0, row0 + 32) of the heads that share a kv head, into a tile.
template <int NQ, int DT>
__device__ __forceinline__ void load_query_rows(AttnTile<NQ, DT, kKvRows> &t, const AttnView &x, const AttnShape &s, int b, int kh, int row0, int end,
                                                bool codes, const ElemFormat &f)
{
    constexpr int kEights = 4 * DT, kAll = kKvRows * kEights;
#pragma unroll
    for (int i = 0; i < (kAll + 255) / 256; ++i) {
        const int n = threadIdx.x + 256 * i, r = n / kEights, col = (n % kEights) * 8, row = row0 + r;
        const int count = row < end ? min(s.dim - col, 8) : 0;
        float v[8];
        if (count > 0) {
            load8_any(x.p, b * x.sb + (row / s.group) * x.st + (kh * s.group + row % s.group) * x.sh + col, count, v, codes, f);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        }
        u32x4 p[NQ];
        bf16_pieces<NQ>(v, p);
        if (n < kAll)
#pragma unroll
            for (int k = 0; k < NQ; ++k) *reinterpret_cast<u32x4 *>(&t.e[k][r][col]) = p[k];
    }
}

// Rows per step with fp16 operands.
template <int DT>
constexpr int kHalfRows = DT == 2 ? 64 : 32;

// Keys whose dK and dV a workgroup adds up over (a part of) the rows that may see them.  Parts end at the same rows on either way of computing
// (fp16 operands or pieces of bf16): the parts of a tile choose between them each for itself.
struct KeyBlock {
    int b, kh, part, k0, key, rows, first, last;
    bool live, used, partial;
    int64_t info;
    AttnSeq seq;
};
template <int DT>
__device__ __forceinline__ KeyBlock key_block(const AttnBwd &a, uint32_t id)
{
    constexpr int step = kHalfRows<DT>;
    const AttnShape &s = a.s;
    KeyBlock k;
    // tiles in parts first (they are the ones with the most rows), then the others
    const uint32_t in_parts = a.part_tiles * a.parts, blocks = in_parts + a.key_tiles - a.part_tiles, n = id % blocks, rest = id / blocks;
    const uint32_t tile = n < in_parts ? n / a.parts : n - in_parts + a.part_tiles, part = n < in_parts ? n % a.parts : 0u;
    const int parts = n < in_parts ? a.parts : 1;
    k.kh = static_cast<int>(rest % s.kv_heads);
    k.b = static_cast<int>(rest / s.kv_heads);
    k.part = static_cast<int>(part);
    k.partial = n < in_parts;
    k.k0 = static_cast<int>(tile) * kKvKeys;
    k.key = k.k0 + static_cast<int>(threadIdx.x >> 6) * 32 + static_cast<int>(threadIdx.x & 31);
    k.seq = attn_seq(s, k.b);
    k.live = k.key < s.k_len;
    k.used = k.key < k.seq.length;
    k.rows = s.q_len * s.group;
    k.info = (static_cast<int64_t>(k.b) * s.kv_heads + k.kh) * a.row_tiles * kRowTile;
    // tokens that may see one of these keys
    int64_t t0 = 0, t1 = s.q_len;
    if (s.causal) t0 = max(t0, static_cast<int64_t>(k.k0) - k.seq.first);
    if (s.window && k.k0 >= s.sinks) {
        t0 = max(t0, static_cast<int64_t>(k.k0) - s.window + 1 - k.seq.first);
        t1 = min(t1, static_cast<int64_t>(k.k0) + kKvKeys - 1 + s.window - k.seq.first);
    }
    if (k.k0 >= k.seq.length) t1 = 0;
    k.first = k.last = 0;
    if (t0 < t1) {                       // in steps, and of these the part
        const int64_t n0 = t0 * s.group / step, n1 = (t1 * s.group + step - 1) / step, all = n1 - n0;
        k.first = static_cast<int>(n0 + all * k.part / parts) * step;
        k.last = static_cast<int>(n0 + all * (k.part + 1) / parts) * step;
    }
    return k;
}

template <int DT>
__device__ __forceinline__ void store_dkv(const AttnBwd &a, const KeyBlock &k, const f32x16 (&dk)[DT], const f32x16 (&dv)[DT], float kscale,
                                          float vscale)
{
    if (!k.live) return;
    const AttnShape &s = a.s;
    const int half = (threadIdx.x & 63) >> 5;
    const int64_t whole = static_cast<int64_t>(s.batch) * a.part_keys * s.kv_heads * s.dim;
    const int64_t at = ((static_cast<int64_t>(k.b) * a.part_keys + k.key) * s.kv_heads + k.kh) * s.dim + k.part * whole;
    const bool part = k.partial;
    void *kout = part ? a.part : const_cast<void *>(a.dk.p), *vout = part ? a.part + a.parts * whole : const_cast<void *>(a.dv.p);
    const int64_t kbase = part ? at : k.b * a.dk.sb + k.key * a.dk.st + k.kh * a.dk.sh;
    const int64_t vbase = part ? at : k.b * a.dv.sb + k.key * a.dv.st + k.kh * a.dv.sh;
    const int result = part ? FMT_RESULT_F32 : a.result;
    store_row<DT>(kout, kbase, half, s.dim, dk, kscale, result, a.f);
    store_row<DT>(vout, vbase, half, s.dim, dv, vscale, result, a.f);
}

template <int DT>
struct DkvShared {
    AttnTile<kPieces, DT, kKvRows> qs, gs;
    float lses[kKvRows], deltas[kKvRows];
};

template <int DT>
__device__ __forceinline__ void dkv_pieces(const AttnBwd &a, uint32_t id, DkvShared<DT> &sh)
{
    constexpr int NQ = kPieces, NP = kProbPieces;
    static_assert(kHalfRows<DT> % kKvRows == 0);
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const KeyBlock key = key_block<DT>(a, id);
    const int b = key.b, kh = key.kh, rows = key.rows;
    const AttnSeq seq = key.seq;
    const int64_t all_rows = info_rows(a);

    u32x4 k[2 * DT][NQ], v[2 * DT][NQ];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half, count = key.used ? min(s.dim - col, 8) : 0;
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = y[j] = 0.0f;
        if (count > 0) {
            load8_any(a.k.p, b * a.k.sb + key.key * a.k.st + kh * a.k.sh + col, count, x, a.codes, a.f);
            load8_any(a.v.p, b * a.v.sb + key.key * a.v.st + kh * a.v.sh + col, count, y, a.codes, a.f);
        }
        bf16_pieces<NQ>(x, k[kk]);
        bf16_pieces<NQ>(y, v[kk]);
    }
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;

    for (int row0 = key.first; row0 < key.last; row0 += kKvRows) {
        __syncthreads();
        load_query_rows<NQ, DT>(sh.qs, a.q, s, b, kh, row0, rows, a.codes, a.f);
        load_query_rows<NQ, DT>(sh.gs, a.go, s, b, kh, row0, rows, a.gcodes, a.f);
        if (threadIdx.x < kKvRows) {
            const int row = row0 + threadIdx.x;
            const bool there = row < rows;
            sh.lses[threadIdx.x] = there ? a.info[kInfoLse2 * all_rows + key.info + row] : INFINITY;
            sh.deltas[threadIdx.x] = there ? a.info[kInfoDelta * all_rows + key.info + row] : 0.0f;
        }
        __syncthreads();
        f32x16 x, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 2 * DT; ++kk) {
            u32x4 f[NQ];
            read_rows(sh.qs, lane & 31, 16 * kk + 8 * half, f);
            x = mfma_pieces<NQ, NQ>(f, k[kk], x);
            read_rows(sh.gs, lane & 31, 16 * kk + 8 * half, f);
            dp = mfma_pieces<NQ, NQ>(f, v[kk], dp);
        }
        const int64_t i0 = static_cast<int64_t>(seq.first) + row0 / s.group;
        const int64_t i1 = static_cast<int64_t>(seq.first) + (min(row0 + kKvRows, rows) - 1) / s.group;
        const bool all = attn_sees_all(s, seq.length, i0, i1, key.k0, key.k0 + kKvKeys);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            float p[8], ds[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = 8 * kb + j, r = 8 * (i / 4) + 4 * half + (i & 3);
                float y = x[i] * s.scale2;
                if (!all && !attn_sees(s, seq.length, seq.first + (row0 + r) / s.group, key.key)) y = -INFINITY;
                p[j] = exp2_fast(y - sh.lses[r]);
                ds[j] = p[j] == 0.0f ? 0.0f : p[j] * (dp[i] - sh.deltas[r]);
            }
            u32x4 pp[NP], dd[NP];
            bf16_pieces<NP>(p, pp);
            bf16_pieces<NP>(ds, dd);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                u32x4 f[NQ];
                read_columns(sh.gs, 16 * kb, 32 * d, lane, f);
                dv[d] = mfma_pieces<NQ, NP>(f, pp, dv[d]);
                read_columns(sh.qs, 16 * kb, 32 * d, lane, f);
                dk[d] = mfma_pieces<NQ, NP>(f, dd, dk[d]);
            }
        }
    }
    store_dkv<DT>(a, key, dk, dv, s.scale, 1.0f);
}

// Both in one launch, workgroups of keys first.
template <int DT>
__global__ __launch_bounds__(256) void attn_bwd_kernel(AttnBwd a)
{
    __shared__ union Shared {
        DqShared<DT> q;
        DkvShared<DT> kv;
        __device__ Shared() {}
    } sh;
    if (blockIdx.x < a.key_blocks) dkv_pieces<DT>(a, xcd_order(blockIdx.x, a.key_blocks), sh.kv);
    else dq_pieces<DT>(a, xcd_order(blockIdx.x - a.key_blocks, a.row_blocks), sh.q);
}

// ---- operands of one fp16 value each, P and dS in NP pieces of fp16
//
// A row of dO is taken times its own power of two, 2^grow, which brings its largest element to [2^14, 2^15): dP and dS of a row carry that
// factor.  dQ loses it at the end.  dK and dV add up rows: there P and dS of a row are taken times 2^(c - grow), with c the smallest grow so far.
//
// P and dS go to fp16 times a power of two of the sum that they enter: of the row in dQ, of the key in dK and dV (both are one lane's, and that of
// the lane 32 on).  It falls, with the sums so far, when a value passes 2^15, and rises when the first values of a row or key lie below kFactorFloor:
// half the step of small fp16 numbers, 2^-25, is then at most 2^-20 of the largest (one piece: 2^-15).  Taken times one factor for a whole tile of rows
// instead, keys that only rows of small dO see lost their P and dS.  (The factor of P costs a product per score.)

// Elements that lost bits on their way to fp16 (below 2^-24 in 11 bits of 1/6/9, for instance) count where they enter a sum of their own channel: of K in dQ, of
// Q in dK, of dO in dV.  A workgroup that reads such elements adds what was cut in a second run over the tiles that hold them, what V lost in dQ's dP with it.
// In other sums over channels what V and dO lost is held against the largest dS of the row or key: it may come to 2^-20 of that, and pieces of bf16 are
// taken otherwise.
//
// What is to know of 32 rows of an operand: the largest |x| as a bit pattern less its last eight bits, there the most elements of a
// row that lost bits (of dO, of V), and in the sign bit whether a second run is wanted.
__device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b)
{
    return max(a & 0x7FFFFF00u, b & 0x7FFFFF00u) | max(a & 0xFFu, b & 0xFFu) | ((a | b) & 0x80000000u);
}
struct Highs {
    uint32_t q = 0, k = 0, v = 0;
};
// The most that dP may have lost, before P, in the units that dS is held in (dO at 2^15, V as it is): of dO, of V.
__device__ __forceinline__ float dp_lost_of_do(const Highs &h) { return static_cast<float>(h.q & 0xFFu) * 0x1p-24f * __uint_as_float(h.v & 0x7FFFFF00u); }
__device__ __forceinline__ float dp_lost_of_v(const Highs &h) { return static_cast<float>(h.v & 0xFFu) * 0x1p-18f; }
// The larger magnitude (NaN stays).
__device__ __forceinline__ float larger(float a, float b, float top)
{
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(a), fabsf(b)), top);
}
constexpr float kFactorMost = 32768.0f;         // what P and dS may be in fp16
constexpr int kKeyFactor = 14;                  // the first exponent of a key's factor: P of 1 fits; of a row's: 0
constexpr int kGrowSpread = 60;                 // rows of dO further apart, in binades, are left to the pieces of bf16
__device__ __forceinline__ int exponent_of(float x) { return static_cast<int>(__float_as_uint(x) >> 23) - 127; }

template <int NP>
constexpr float kFactorFloor = NP == 2 ? 0x1p-5f : 0x1p-10f;

// Whether a factor has to change: the larger of its largest products has passed, or is NaN, or the smaller one is small and there is room.
// (dK's dS share the factor of dV's P.)  What is below `least` is taken for nothing: with a factor that brought it up, other products would overflow
// (a row's dP comes to 2^38 at most, in the units that dS is held in, and is multiplied by the factor before P).
constexpr float kRowLeast = 0x1p-60f, kKeyLeast = 0x1p-80f;
constexpr int kRowMost = 80, kKeyMost = 104;         // exponents that factors do not pass
template <int NP>
__device__ __forceinline__ bool factor_off(float high, float low, float least)
{
    return !(high <= kFactorMost) || (low < kFactorFloor<NP> && low > least && high < 1024.0f);
}

// By how many binades the factors of a wave fall (rise: negative).  When one changes, others that are low rise as well, and those that have seen
// nothing go with one that rises, so that few changes follow.  room: how far they may rise.
__device__ __forceinline__ int factor_fall(float high, float low, float least, int room)
{
    int fall = high > kFactorMost ? exponent_of(high) - 11 : low > least && low < 64.0f ? min(max(exponent_of(low) - 9, exponent_of(high) - 11), 0) : 0;
    if (!(high < INFINITY)) fall = 0;
    const uint64_t rising = __ballot(fall < 0);
    if (rising) {
        const int one = __builtin_amdgcn_readlane(fall, __builtin_ctzll(rising));
        if (high <= least) fall = max(one, -20);
    }
    return max(fall, -room);
}
// The smaller of two largest products, where the second is not nothing.
__device__ __forceinline__ float smaller(float a, float b) { return b > kKeyLeast ? fminf(a, b) : a; }

// x times 2^n for any n that ends among the normal numbers: what is left of the factor for the last product.
template <int DT>
__device__ __forceinline__ float bring_down(f32x16 (&x)[DT], int n, float last)
{
    const float first = ldexpf(1.0f, n / 2);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[d][i] *= first;
    return ldexpf(last, n - n / 2);
}
template <int DT>
__device__ __forceinline__ void times(f32x16 (&x)[DT], float factor)
{
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[d][i] *= factor;
}

// Where attn_pack_kernel left them for one (batch, kv head).
struct PackHighs {
    const uint32_t *q, *k, *v;
    __device__ __forceinline__ PackHighs(const AttnBwd &a, uint32_t bkh)
    {
        const uint32_t rows = a.row_tiles * (kRowTile / kPackRows), keys = a.key_tiles * (kKvKeys / kPackRows), all = a.s.kv_heads * a.s.batch;
        q = a.highs + bkh * rows;
        k = a.highs + all * rows + bkh * keys;
        v = k + all * keys;
    }
    __device__ __forceinline__ uint32_t of(const uint32_t *p, int first, int count) const
    {
        uint32_t h = 0;
        for (int i = 0; i < count / kPackRows; ++i) h = join(h, p[first / kPackRows + i]);
        return h;
    }
};

// Whether a workgroup has to be computed with bf16 pieces: in all of its threads.
__device__ __forceinline__ bool half_flags(const AttnBwd &a, const Highs &h, bool bad)
{
    if (a.check) {                                     // q, k and v are the same in the whole workgroup
        const uint32_t scores = max(h.q & 0x7FFFFF00u, h.k & 0x7FFFFF00u);
        bad |= scores >= __float_as_uint(a.limit) || (h.v & 0x7FFFFF00u) >= __float_as_uint(ldexpf(1.0f, kHalfLimit));
    }
    return __syncthreads_or(bad);
}

// Sixteen bytes per thread and step of a tile of whole rows.
template <int DT, int ROWS>
struct TileLoad {
    static constexpr int kLoads = ROWS * 4 * DT / 256;
    u32x4 r[kLoads];
    __device__ __forceinline__ void fetch(const uint16_t *rows)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) r[i] = reinterpret_cast<const u32x4 *>(rows)[threadIdx.x + 256 * i];
    }
    __device__ __forceinline__ void put(AttnTile<1, DT, ROWS> &t) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int n = threadIdx.x + 256 * i;
            *reinterpret_cast<u32x4 *>(&t.e[0][n / (4 * DT)][(n % (4 * DT)) * 8]) = r[i];
        }
    }
};

// Second runs cost as much as a first: one channel of K or V of 2^-30, so that every tile has some: 4096 tokens, 8 heads of 128, 1/6/9: 436 -> 1147 us,
// and 2319 with pieces of bf16 throughout (V of 200).  A few lost elements cost a few microseconds at the end of the workgroups that read them.
//
// What was cut of tokens [first, first + ROWS) of one head (load_tokens).
template <int DT, int ROWS>
__device__ __forceinline__ void load_rests(AttnTile<1, DT, ROWS> &t, const void *x, int64_t base, int64_t stride, int first, int end, int dim, bool codes,
                                           const ElemFormat &f, float up)
{
    constexpr int kEights = 4 * DT;
    bool ignore = false;
#pragma unroll 2
    for (int i = 0; i < ROWS * kEights / 256; ++i) {
        const int n = threadIdx.x + 256 * i, row = n / kEights, col = (n % kEights) * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        if (first + row < end && col < dim) load8_any(x, base + (first + row) * stride + col, min(dim - col, 8), v, codes, f);
        *reinterpret_cast<u32x4 *>(&t.e[0][row][col]) = half_rest(v, up, ignore);
    }
}

template <int DT>
struct DqHalfShared {
    AttnTile<1, DT, kKeyTile> ks[2], vs[2];
};

// The same number, as far as the compiler knows another one: what is computed from it again need not be kept.
__device__ __forceinline__ uint32_t opaque(uint32_t id)
{
    asm volatile("" : "+v"(id));
    return __builtin_amdgcn_readfirstlane(id);
}

// What V lost, in dS, and then what K lost, times 2^24: over the tiles concerned.
template <int NP, int DT>
__device__ __forceinline__ void dq_rests(const AttnBwd &a, uint32_t id, const Highs &high, DqHalfShared<DT> &sh, f32x16 (&dq)[DT], int factor, float &most,
                                         bool &bad)
{
    constexpr int DP = 32 * DT;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const RowBlock r = row_block(a, id);
    const uint32_t bkh = r.b * s.kv_heads + r.kh;
    const PackHighs highs(a, bkh);
    const int64_t all_rows = info_rows(a), kbase = r.b * a.k.sb + r.kh * a.k.sh, vbase = r.b * a.v.sb + r.kh * a.v.sh;
    const uint16_t *keys = a.kh + static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys * DP, *values = a.vh + static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys * DP;
    const AttnTiles tiles = attn_tiles(s, r.seq.length, r.i0, r.i1, kKeyTile);
    const float lse2 = a.info[kInfoLse2 * all_rows + r.info], delta = a.info[kInfoScaledDelta * all_rows + r.info];
    const float scale2 = s.scale == 0.0f ? 1.0f : fabsf(s.scale2) / (a.up * a.up);
    const float dp_by = ldexpf(1.0f / a.up, factor), delta_by = ldexpf(delta, factor);
    const AttnKeys sees = attn_keys(s, r.seq.length, r.pos);
#pragma unroll 1
    for (int of_k = high.v & 0xFFu ? 0 : 1; of_k < (high.k >> 31 ? 2 : 1); ++of_k) {
        if (of_k) times<DT>(dq, kRestUp);
#pragma unroll 1
        for (int n = 0; n < tiles.count(); ++n) {
            const int tile = tiles.at(n), k0 = tile * kKeyTile;
            if (!(of_k ? highs.of(highs.k, k0, kKeyTile) >> 31 : highs.of(highs.v, k0, kKeyTile) & 0xFFu)) continue;
            TileLoad<DT, kKeyTile> k_load, v_load;
            k_load.fetch(keys + static_cast<int64_t>(tile) * kKeyTile * DP);
            v_load.fetch(values + static_cast<int64_t>(tile) * kKeyTile * DP);
            k_load.put(sh.ks[0]);
            v_load.put(sh.vs[0]);
            load_rests<DT, kKeyTile>(sh.ks[1], a.k.p, kbase, a.k.st, k0, r.seq.length, s.dim, a.codes, a.f, a.up);
            load_rests<DT, kKeyTile>(sh.vs[1], a.v.p, vbase, a.v.st, k0, r.seq.length, s.dim, a.codes, a.f, a.up);
            __syncthreads();
#pragma unroll 1
            for (int kt = 0; kt < 2; ++kt) {
                f32x16 x, dp, more;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = dp[i] = more[i] = 0.0f;
#pragma unroll
                for (int kk = 0; kk < 2 * DT; ++kk) {
                    const u32x4 q = *reinterpret_cast<const u32x4 *>(a.qh + r.info * DP + 16 * kk + 8 * half);
                    const u32x4 go = *reinterpret_cast<const u32x4 *>(a.gh + r.info * DP + 16 * kk + 8 * half);
                    u32x4 f[1];
                    read_rows(sh.ks[0], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                    x = mfma_f16(f[0], q, x);
                    read_rows(sh.vs[0], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                    dp = mfma_f16(f[0], go, dp);
                    read_rows(sh.vs[1], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                    more = mfma_f16(f[0], go, more);
                }
                attn_hide(sees, k0 + 32 * kt + 4 * half, x);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = exp2_fast(fmaf(x[i], scale2, -lse2)), rest = more[i] * (1.0f / kRestUp);
                    x[i] = p * (of_k ? fmaf(dp[i] + rest, dp_by, -delta_by) : rest * dp_by);
                }
                if (!of_k) {
#pragma unroll
                    for (int i = 0; i < 16; i += 2) most = larger(x[i], x[i + 1], most);
                }
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    float ds[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) ds[j] = x[8 * kb + j];
                    u32x4 pp[NP];
                    f16_pieces<NP>(ds, pp);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        u32x4 f[1];
                        read_columns(sh.ks[of_k], 32 * kt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                        for (int w = NP - 1; w >= 0; --w) dq[d] = mfma_f16(f[0], pp[w], dq[d]);
                    }
                }
            }
            __syncthreads();
        }
        if (of_k) times<DT>(dq, 1.0f / kRestUp);
    }
    // the factor is that of what there was without the rests
    const float largest = __builtin_elementwise_maximum(most, __shfl_xor(most, 32));
    bad |= !(largest <= kFactorMost) || (largest > kRowLeast && largest < kFactorFloor<NP>);
}

// Returns whether the workgroup has to be computed with bf16 pieces.
template <int NP, int DT>
__device__ __forceinline__ bool dq_half(const AttnBwd &a, uint32_t id, DqHalfShared<DT> &sh)
{
    constexpr int DP = 32 * DT;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const RowBlock r = row_block(a, id);
    const uint32_t bkh = r.b * s.kv_heads + r.kh;
    const PackHighs highs(a, bkh);
    const int64_t all_rows = info_rows(a);
    const uint16_t *keys = a.kh + static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys * DP, *values = a.vh + static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys * DP;
    const AttnTiles tiles = attn_tiles(s, r.seq.length, r.i0, r.i1, kKeyTile);
    const int count = tiles.count();
    Highs high;
    high.q = highs.of(highs.q, r.row0, kRowTile);
    TileLoad<DT, kKeyTile> kr, vr;
    if (count > 0) {
        kr.fetch(keys + static_cast<int64_t>(tiles.at(0)) * kKeyTile * DP);
        vr.fetch(values + static_cast<int64_t>(tiles.at(0)) * kKeyTile * DP);
    }
    const float lse2 = a.info[kInfoLse2 * all_rows + r.info], delta = a.info[kInfoScaledDelta * all_rows + r.info], grow = a.info[kInfoGrow * all_rows + r.info];
    u32x4 q[2 * DT], go[2 * DT];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        q[kk] = *reinterpret_cast<const u32x4 *>(a.qh + r.info * DP + 16 * kk + 8 * half);
        go[kk] = *reinterpret_cast<const u32x4 *>(a.gh + r.info * DP + 16 * kk + 8 * half);
    }
    f32x16 dq[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.0f;
    const float scale2 = s.scale == 0.0f ? 1.0f : fabsf(s.scale2) / (a.up * a.up), down = 1.0f / a.up;
    const AttnKeys sees = attn_keys(s, r.seq.length, r.pos);
    bool bad = false;
    int factor = 0;
    float dp_by = down, delta_by = delta, most = 0.0f;
    for (int n = 0; n < count; ++n) {
        const int tile = tiles.at(n), k0 = tile * kKeyTile, buf = n & 1;
        kr.put(sh.ks[buf]);
        vr.put(sh.vs[buf]);
        high.k = join(high.k, highs.of(highs.k, k0, kKeyTile));
        high.v = join(high.v, highs.of(highs.v, k0, kKeyTile));
        __syncthreads();
        if (n + 1 < count) {
            kr.fetch(keys + static_cast<int64_t>(tiles.at(n + 1)) * kKeyTile * DP);
            vr.fetch(values + static_cast<int64_t>(tiles.at(n + 1)) * kKeyTile * DP);
        }
        const bool all = attn_sees_all(s, r.seq.length, r.i0, r.i1, k0, k0 + kKeyTile);
#pragma unroll 1
        for (int kt = 0; kt < 2; ++kt) {
            f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                u32x4 f[1];
                read_rows(sh.ks[buf], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                x = mfma_f16(f[0], q[kk], x);
                read_rows(sh.vs[buf], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                dp = mfma_f16(f[0], go[kk], dp);
            }
            if (!all) attn_hide(sees, k0 + 32 * kt + 4 * half, x);
            float top = most;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = exp2_fast(fmaf(x[i], scale2, -lse2)) * fmaf(dp[i], dp_by, -delta_by);
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = larger(x[i], x[i + 1], top);
            if (__builtin_expect(__any(factor_off<NP>(top, top, kRowLeast)), 0)) {
                const float both = __builtin_elementwise_maximum(top, __shfl_xor(top, 32));
                const int fall = factor_fall(both, both, kRowLeast, kRowMost - factor);
                bad |= !(both < INFINITY);
                factor -= fall;
                dp_by = ldexpf(down, factor);
                delta_by = ldexpf(delta, factor);
                const float by = ldexpf(1.0f, -fall);
                times<DT>(dq, by);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] *= by;
                top = both * by;                                       // (the same in both lanes: what is small in one need not be in the other)
            }
            most = top;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float ds[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) ds[j] = x[8 * kb + j];
                u32x4 pp[NP];
                f16_pieces<NP>(ds, pp);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[1];
                    read_columns(sh.ks[buf], 32 * kt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                    for (int w = NP - 1; w >= 0; --w) dq[d] = mfma_f16(f[0], pp[w], dq[d]);
                }
            }
        }
    }
    if (r.live && lse2 < INFINITY && grow != kNoRow) {
        const float largest = __builtin_elementwise_maximum(most, __shfl_xor(most, 32));
        // (beside a delta 2^24 times as large dP loses no more than it does in fp32; dS of a row that sees one key is nothing but rounding)
        bad |= ldexpf(dp_lost_of_do(high), factor + 20) > largest && dp_lost_of_do(high) > fabsf(delta) * 0x1p-24f;
    }
    if (__builtin_expect(half_flags(a, high, bad), 0)) return true;
    if (__builtin_expect((high.k >> 31) | (high.v & 0xFFu), 0)) {             // the same in the whole workgroup
        dq_rests<NP, DT>(a, opaque(id), high, sh, dq, factor, most, bad);
        if (__syncthreads_or(bad)) return true;
    }
    const float last = bring_down<DT>(dq, grow == kNoRow ? 0 : -static_cast<int>(grow) - factor, s.scale * down);
    store_dq<DT>(a, r, dq, last);
    return false;
}

template <int DT>
struct DkvHalfShared {
    AttnTile<1, DT, kHalfRows<DT>> qs[2], gs[2];
    alignas(16) float lse[2][kHalfRows<DT>], delta[2][kHalfRows<DT>];
    float least[2];
};

// What was cut of Q and dO, rows [row0, row0 + kHalfRows) of the heads that share a kv head.
template <int DT>
__device__ __forceinline__ void load_row_rests(const AttnBwd &a, AttnTile<1, DT, kHalfRows<DT>> &qs, AttnTile<1, DT, kHalfRows<DT>> &gs, const KeyBlock &key,
                                               int row0)
{
    constexpr int kEights = 4 * DT;
    const AttnShape &s = a.s;
    bool ignore = false;
#pragma unroll
    for (int i = 0; i < kHalfRows<DT> * kEights / 256; ++i) {
        const int n = threadIdx.x + 256 * i, r = n / kEights, col = (n % kEights) * 8, row = row0 + r;
        float q[8], g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = g[j] = 0.0f;
        if (row < key.rows && col < s.dim) {
            const RowAt at = row_at(row, s.group);
            const int count = min(s.dim - col, 8), head = key.kh * s.group + at.g;
            load8_any(a.q.p, key.b * a.q.sb + at.t * a.q.st + head * a.q.sh + col, count, q, a.codes, a.f);
            load8_any(a.go.p, key.b * a.go.sb + at.t * a.go.st + head * a.go.sh + col, count, g, a.gcodes, a.f);
            const float grow = a.info[kInfoGrow * info_rows(a) + key.info + row];
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = ldexpf(g[j], grow == kNoRow ? 0 : static_cast<int>(grow));
        }
        *reinterpret_cast<u32x4 *>(&qs.e[0][r][col]) = half_signed(half_rest(q, a.up, ignore), s.scale);
        *reinterpret_cast<u32x4 *>(&gs.e[0][r][col]) = half_rest(g, 1.0f, ignore);
    }
}

// Rows that see a lane's key.
struct SeenRows {
    int first;
    uint32_t count;
};
__device__ __forceinline__ SeenRows rows_that_see(const AttnShape &s, const KeyBlock &key)
{
    SeenRows seen{0, 0};
    if (key.used) {
        int64_t t0 = 0, t1 = s.q_len;
        if (s.causal) t0 = max(t0, static_cast<int64_t>(key.key) - key.seq.first);
        if (s.window && key.key >= s.sinks) {
            t0 = max(t0, static_cast<int64_t>(key.key) - s.window + 1 - key.seq.first);
            t1 = min(t1, static_cast<int64_t>(key.key) + s.window - key.seq.first);
        }
        if (t0 < t1) seen = SeenRows{static_cast<int>(t0 * s.group), static_cast<uint32_t>((t1 - t0) * s.group)};
    }
    return seen;
}

// What Q and dO lost, times 2^24, in dK and dV: over the tiles concerned.
template <int NP, int DT>
__device__ __forceinline__ void dkv_rests(const AttnBwd &a, uint32_t id, DkvHalfShared<DT> &sh, f32x16 (&dk)[DT], f32x16 (&dv)[DT], float least, float by)
{
    constexpr int kRows = kHalfRows<DT>, DP = 32 * DT;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const KeyBlock key = key_block<DT>(a, id);
    const uint32_t bkh = key.b * s.kv_heads + key.kh;
    const PackHighs highs(a, bkh);
    const int64_t all_rows = info_rows(a), mine = (static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys + key.key) * DP + 8 * half;
    const uint16_t *queries = a.qh + key.info * DP, *gradients = a.gh + key.info * DP;
    const float scale2 = s.scale == 0.0f ? 1.0f : fabsf(s.scale2) / (a.up * a.up), down17 = 0x1p-17f / a.up;
    const SeenRows seen = rows_that_see(s, key);
    times<DT>(dk, kRestUp);
    times<DT>(dv, kRestUp);
#pragma unroll 1
    for (int row0 = key.first; row0 < key.last; row0 += kRows) {
        if (!(highs.of(highs.q, row0, kRows) >> 31)) continue;
        TileLoad<DT, kRows> q_load, g_load;
        q_load.fetch(queries + static_cast<int64_t>(row0) * DP);
        g_load.fetch(gradients + static_cast<int64_t>(row0) * DP);
        q_load.put(sh.qs[0]);
        g_load.put(sh.gs[0]);
        load_row_rests<DT>(a, sh.qs[1], sh.gs[1], key, row0);
        if (threadIdx.x < kRows) {
            const int64_t at = key.info + row0 + threadIdx.x;
            const float grow = a.info[kInfoGrow * all_rows + at];
            sh.lse[0][threadIdx.x] = grow == kNoRow ? INFINITY : a.info[kInfoLse2 * all_rows + at] - (least - grow);
            sh.delta[0][threadIdx.x] = a.info[kInfoScaledDelta * all_rows + at] * 0x1p-17f;
        }
        __syncthreads();
#pragma unroll 1
        for (int rt = 0; rt < kRows / 32; ++rt) {
            f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                const u32x4 k = *reinterpret_cast<const u32x4 *>(a.kh + mine + 16 * kk), v = *reinterpret_cast<const u32x4 *>(a.vh + mine + 16 * kk);
                u32x4 f[1];
                read_rows(sh.qs[0], 32 * rt + (lane & 31), 16 * kk + 8 * half, f);
                x = mfma_f16(f[0], k, x);
                read_rows(sh.gs[0], 32 * rt + (lane & 31), 16 * kk + 8 * half, f);
                dp = mfma_f16(f[0], v, dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 32 * rt + 8 * (i / 4) + 4 * half + (i & 3);
                const float score = static_cast<uint32_t>(row0 + row - seen.first) < seen.count ? x[i] : -INFINITY;
                x[i] = exp2_fast(fmaf(score, scale2, -sh.lse[0][row])) * by;
                dp[i] = x[i] * fmaf(dp[i], down17, -sh.delta[0][row]);
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float p[8], ds[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = x[8 * kb + j], ds[j] = dp[8 * kb + j];
                u32x4 pp[NP], dd[NP];
                f16_pieces<NP>(p, pp);
                f16_pieces<NP>(ds, dd);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[1];
                    read_columns(sh.gs[1], 32 * rt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                    for (int w = NP - 1; w >= 0; --w) dv[d] = mfma_f16(f[0], pp[w], dv[d]);
                    read_columns(sh.qs[1], 32 * rt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                    for (int w = NP - 1; w >= 0; --w) dk[d] = mfma_f16(f[0], dd[w], dk[d]);
                }
            }
        }
        __syncthreads();
    }
    times<DT>(dk, 1.0f / kRestUp);
    times<DT>(dv, 1.0f / kRestUp);
}

template <int NP, int DT>
__device__ __forceinline__ bool dkv_half(const AttnBwd &a, uint32_t id, DkvHalfShared<DT> &sh)
{
    constexpr int kRows = kHalfRows<DT>, DP = 32 * DT;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const KeyBlock key = key_block<DT>(a, id);
    const uint32_t bkh = key.b * s.kv_heads + key.kh;
    const PackHighs highs(a, bkh);
    const int64_t all_rows = info_rows(a);
    const uint16_t *queries = a.qh + key.info * DP, *gradients = a.gh + key.info * DP;
    Highs high;
    high.k = highs.of(highs.k, key.k0, kKvKeys);
    high.v = highs.of(highs.v, key.k0, kKvKeys);
    TileLoad<DT, kRows> qr, gr;
    float info[3];
    auto fetch = [&](int row0) __attribute__((always_inline)) {
        qr.fetch(queries + static_cast<int64_t>(row0) * DP);
        gr.fetch(gradients + static_cast<int64_t>(row0) * DP);
        const int64_t at = key.info + row0 + (threadIdx.x & (kRows - 1));
        info[0] = a.info[kInfoLse2 * all_rows + at];
        info[1] = a.info[kInfoScaledDelta * all_rows + at];
        info[2] = a.info[kInfoGrow * all_rows + at];
    };
    if (key.first < key.last) fetch(key.first);
    u32x4 k[2 * DT], v[2 * DT];
    const int64_t mine = (static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys + key.key) * DP + 8 * half;
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        k[kk] = *reinterpret_cast<const u32x4 *>(a.kh + mine + 16 * kk);
        v[kk] = *reinterpret_cast<const u32x4 *>(a.vh + mine + 16 * kk);
    }
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;
    const float scale2 = s.scale == 0.0f ? 1.0f : fabsf(s.scale2) / (a.up * a.up), down = 1.0f / a.up;
    const float down17 = down * 0x1p-17f;
    const SeenRows seen = rows_that_see(s, key);
    float least = kNoRow, running = kNoRow, widest = -kNoRow;      // the smallest grow: of the sums, and (wave 0) of the rows read so far; the largest of those
    bool bad = false;
    int factor = kKeyFactor;
    float by = ldexpf(1.0f, factor), most = 0.0f, most_ds = 0.0f;        // the largest P and dS so far, as the sums are held
    int buf = 0;
    for (int row0 = key.first; row0 < key.last; row0 += kRows, buf ^= 1) {
        qr.put(sh.qs[buf]);
        gr.put(sh.gs[buf]);
        high.q = join(high.q, highs.of(highs.q, row0, kRows));
        if (threadIdx.x < 64) {
            float low = info[2], wide = info[2] == kNoRow ? -kNoRow : info[2];
#pragma unroll
            for (int w = 32; w > 0; w >>= 1) {
                low = fminf(low, __shfl_xor(low, w));
                wide = fmaxf(wide, __shfl_xor(wide, w));
            }
            running = fminf(running, low);
            widest = fmaxf(widest, wide);
            if (threadIdx.x < kRows) {
                // P of the row times 2^(c - grow) comes out of the exponential (a row of zeros has none), and delta goes with it
                sh.lse[buf][threadIdx.x] = info[2] == kNoRow ? INFINITY : info[0] - (running - info[2]);
                sh.delta[buf][threadIdx.x] = info[1] * 0x1p-17f;
            }
            if (threadIdx.x == 0) sh.least[buf] = running;
        }
        __syncthreads();
        if (row0 + kRows < key.last) fetch(row0 + kRows);
        const float next = sh.least[buf];
        if (next < least) {                                        // the same in the whole workgroup
            // what the sums hold falls with c, but no further than to a largest P of 2^3: from there on the factor rises instead
            const int by_now = least == kNoRow ? 0 : static_cast<int>(least - next);
            const float both = fmaxf(most, __shfl_xor(most, 32));
            const int fall = both > 0.0f ? min(by_now, max(max(exponent_of(both) - 3, factor + by_now - kKeyMost), 0)) : by_now;
            least = next;
            factor += by_now - fall;
            by = ldexpf(1.0f, factor);
            const float lower = ldexpf(1.0f, -fall);
            times<DT>(dk, lower);
            times<DT>(dv, lower);
            most *= lower;
            most_ds *= lower;
        }
        const int64_t i0 = static_cast<int64_t>(key.seq.first) + row0 / s.group;
        const int64_t i1 = static_cast<int64_t>(key.seq.first) + (min(row0 + kRows, key.rows) - 1) / s.group;
        const bool all = attn_sees_all(s, key.seq.length, i0, i1, key.k0, key.k0 + kKvKeys);
#pragma unroll 1
        for (int rt = 0; rt < kRows / 32; ++rt) {
            f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                u32x4 f[1];
                read_rows(sh.qs[buf], 32 * rt + (lane & 31), 16 * kk + 8 * half, f);
                x = mfma_f16(f[0], k[kk], x);
                read_rows(sh.gs[buf], 32 * rt + (lane & 31), 16 * kk + 8 * half, f);
                dp = mfma_f16(f[0], v[kk], dp);
            }
            if (!all) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[i] = static_cast<uint32_t>(row0 + 32 * rt + 8 * (i / 4) + 4 * half + (i & 3) - seen.first) < seen.count ? x[i] : -INFINITY;
            }
            float top = most, top_ds = most_ds;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int row = 32 * rt + 8 * g + 4 * half;
                const f32x4 lse = *reinterpret_cast<const f32x4 *>(&sh.lse[buf][row]), delta = *reinterpret_cast<const f32x4 *>(&sh.delta[buf][row]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[4 * g + j] = exp2_fast(fmaf(x[4 * g + j], scale2, -lse[j])) * by;
                    dp[4 * g + j] = x[4 * g + j] * fmaf(dp[4 * g + j], down17, -delta[j]);
                }
                top = larger(x[4 * g], x[4 * g + 1], larger(x[4 * g + 2], x[4 * g + 3], top));
                top_ds = larger(dp[4 * g], dp[4 * g + 1], larger(dp[4 * g + 2], dp[4 * g + 3], top_ds));
            }
            if (__builtin_expect(__any(factor_off<NP>(__builtin_elementwise_maximum(top, top_ds), smaller(top, top_ds), kKeyLeast)), 0)) {
                const float both = __builtin_elementwise_maximum(top, __shfl_xor(top, 32)), both_ds = __builtin_elementwise_maximum(top_ds, __shfl_xor(top_ds, 32));
                const float higher = __builtin_elementwise_maximum(both, both_ds);
                const int fall = factor_fall(higher, smaller(both, both_ds), kKeyLeast, kKeyMost - factor);
                bad |= !(higher < INFINITY);
                factor -= fall;
                by = ldexpf(1.0f, factor);
                const float lower = ldexpf(1.0f, -fall);
                times<DT>(dk, lower);
                times<DT>(dv, lower);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[i] *= lower;
                    dp[i] *= lower;
                }
                top = both * lower;                                    // (the same in both lanes: what is small in one need not be in the other)
                top_ds = both_ds * lower;
            }
            most = top;
            most_ds = top_ds;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float p[8], ds[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = x[8 * kb + j], ds[j] = dp[8 * kb + j];
                u32x4 pp[NP], dd[NP];
                f16_pieces<NP>(p, pp);
                f16_pieces<NP>(ds, dd);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[1];
                    read_columns(sh.gs[buf], 32 * rt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                    for (int w = NP - 1; w >= 0; --w) dv[d] = mfma_f16(f[0], pp[w], dv[d]);
                    read_columns(sh.qs[buf], 32 * rt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                    for (int w = NP - 1; w >= 0; --w) dk[d] = mfma_f16(f[0], dd[w], dk[d]);
                }
            }
        }
    }
    // too small beside one another for one factor: V of the key's rows is tiny or large altogether, or their dS all rounding
    most = __builtin_elementwise_maximum(most, __shfl_xor(most, 32));
    most_ds = __builtin_elementwise_maximum(most_ds, __shfl_xor(most_ds, 32));
    // A row's only key has P = 1 and dP = delta: its dS is the rounding of 0, and has nothing to keep (one token, 12 heads of 40: 48 -> 31 us).
    const bool only = key.seq.length == 1 || (s.window == 1 && s.sinks == 0);
    const float low = only ? most : smaller(most, most_ds);
    bad |= widest - running > static_cast<float>(kGrowSpread) || (low > kKeyLeast && low < kFactorFloor<NP>);
    bad |= most * (dp_lost_of_do(high) + dp_lost_of_v(high)) * 0x1p3f > most_ds;      // P dp_lost 2^-17 2^20
    if (__builtin_expect(half_flags(a, high, bad), 0)) return true;
    if (__builtin_expect(high.q >> 31, 0)) dkv_rests<NP, DT>(a, opaque(id), sh, dk, dv, least, by);      // the same in the whole workgroup
    const int lose = least == kNoRow ? 0 : -static_cast<int>(least) - factor;
    const float klast = bring_down<DT>(dk, lose, fabsf(s.scale) * down * 131072.0f), vlast = bring_down<DT>(dv, lose, 1.0f);
    store_dkv<DT>(a, key, dk, dv, klast, vlast);
    return false;
}

template <int NP, int DT>
__global__ __launch_bounds__(256, DT == 2 ? 2 : 1) void attn_bwd_half_kernel(AttnBwd a)
{
    __shared__ union Shared {
        DqHalfShared<DT> q;
        DkvHalfShared<DT> kv;
        DqShared<DT> q_pieces;
        DkvShared<DT> kv_pieces;
        __device__ Shared() {}
    } sh;
    if (blockIdx.x < a.key_blocks) {
        const uint32_t id = xcd_order(blockIdx.x, a.key_blocks);
        if (__builtin_expect(dkv_half<NP, DT>(a, id, sh.kv), 0)) dkv_pieces<DT>(a, opaque(id), sh.kv_pieces);
    } else {
        const uint32_t id = xcd_order(blockIdx.x - a.key_blocks, a.row_blocks);
        if (__builtin_expect(dq_half<NP, DT>(a, id, sh.q), 0)) dq_pieces<DT>(a, opaque(id), sh.q_pieces);
    }
}

}  // namespace

template <int DT>
void run_attention_bwd(const AttnBwd &a, bool half, bool two, dim3 blocks, hipStream_t stream)
{
    if (half && two) attn_bwd_half_kernel<2, DT><<<blocks, dim3(256), 0, stream>>>(a);
    else if (half) attn_bwd_half_kernel<1, DT><<<blocks, dim3(256), 0, stream>>>(a);
    else attn_bwd_kernel<DT><<<blocks, dim3(256), 0, stream>>>(a);
}

}  // namespace fmt
