// Attention, backward (fmt_attention.h has the mathematics and the layouts).
//
// P is made again from Q, K and lse.  Two kernels: one takes rows and adds up dQ over keys, the other takes keys and adds up dK and dV over
// rows, so that every sum is in one workgroup's accumulators, in a fixed order, at the price of S and dP twice (7 products instead of 5).
#include <algorithm>
#include <type_traits>

#include "fmt_attention.h"

namespace fmt {

namespace {

struct AttnBwd {
    AttnShape s;
    AttnView q, k, v, o, go, dq, dk, dv;
    const float *lse;
    float *info;              // what the products need of a row, [4][batch][kv_heads][row_tiles * 128]: kInfo*
    uint16_t *qh, *gh;        // fp16 operands: [batch][kv_heads][row_tiles * 128][32 DT] Q and dO, zero past the last row and column,
    uint16_t *kh, *vh;        // [batch][kv_heads][key_tiles * 128][32 DT] K and V, zero past the sequence's length
    uint32_t *highs;          // the largest |x| of each 32 rows of Q, then of each 32 keys of K, then of V
    float *part;              // parts > 1: [2][parts][batch][k_len][kv_heads][dim] of dK, dV
    uint32_t *flags;          // per workgroup: whether it is left to the pieces of bf16; or nullptr
    float up;                 // what the fp16 operands are multiplied by
    bool check;               // whether that has a limit
    bool codes, gcodes;       // how q, k and v, and o and go, are stored
    int32_t parts;            // parts of the rows that a tile of keys adds up
    uint32_t key_tiles, row_tiles, key_blocks, row_blocks;
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

__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *shared)
{
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), w)));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    return max(max(shared[0], shared[1]), max(shared[2], shared[3]));
}

// What the products need: of 32 rows delta = sum over the head's columns of R(dO) O, lse, and with HALF R(Q) and R(dO) as fp16 operands; with HALF
// also of 32 keys R(K) and R(V).  4 DT lanes per row, 8 columns each.  One pass over the tensors, whose tiles are then read many times.
template <int DT, bool HALF>
__global__ __launch_bounds__(256) void attn_pack_kernel(AttnBwd a)
{
    __shared__ uint32_t shared[4];
    constexpr int kEights = 4 * DT, kStep = 256 / kEights;
    const AttnShape &s = a.s;
    const uint32_t row_packs = a.row_tiles * (kRowTile / kPackRows), key_packs = a.key_tiles * (kKvKeys / kPackRows);
    const uint32_t row_blocks = row_packs * s.kv_heads * s.batch;
    const int col = (threadIdx.x % kEights) * 8, in = threadIdx.x / kEights, count = min(s.dim - col, 8);
    const int64_t all = info_rows(a);
    if (blockIdx.x < row_blocks) {
        const uint32_t tile = blockIdx.x % row_packs, bkh = blockIdx.x / row_packs;
        const int kh = static_cast<int>(bkh % s.kv_heads), b = static_cast<int>(bkh / s.kv_heads), rows = s.q_len * s.group;
        ElemFormat whole = a.f;
        if (!a.gcodes) whole.codec = kCodecNone;                   // O is taken as it is
        uint32_t high_q = 0;
#pragma unroll 1
        for (int r = in; r < kPackRows; r += kStep) {
            const int row = static_cast<int>(tile) * kPackRows + r;
            const int64_t at = static_cast<int64_t>(bkh) * a.row_tiles * kRowTile + row;
            const RowAt where = row_at(row, s.group);
            const int head = kh * s.group + where.g;
            float g[8], o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = o[j] = 0.0f;
            const bool there = row < rows && count > 0;
            if (there) {
                load8_any(a.go.p, b * a.go.sb + where.t * a.go.st + head * a.go.sh + col, count, g, a.gcodes, a.f);
                load8_any(a.o.p, b * a.o.sb + where.t * a.o.st + head * a.o.sh + col, count, o, a.gcodes, whole);
            }
            float sum = 0.0f;
            uint32_t high = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum = fmaf(g[j], o[j], sum);
                high = max(high, __float_as_uint(g[j]) & 0x7FFFFFFFu);
            }
#pragma unroll
            for (int w = kEights / 2; w > 0; w >>= 1) {
                sum += __shfl_xor(sum, w);
                high = max(high, static_cast<uint32_t>(__shfl_xor(static_cast<int>(high), w)));
            }
            const int grow = min(max(138 - static_cast<int>(high >> 23), -120), 120);      // 11 - the exponent of the largest
            if (col == 0) {
                const float lse = row < rows ? a.lse[(static_cast<int64_t>(b) * s.heads + head) * s.q_len + where.t] : -INFINITY;
                a.info[kInfoLse2 * all + at] = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
                a.info[kInfoDelta * all + at] = sum;
                a.info[kInfoGrow * all + at] = high == 0u ? kNoRow : static_cast<float>(grow);
                // (an infinity or NaN in dO makes NaN of the row, and so of the check on dS)
                a.info[kInfoScaledDelta * all + at] = high >= 0x7F800000u ? NAN : ldexpf(sum, grow);
            }
            if constexpr (HALF) {
                f16x8 h;
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = static_cast<_Float16>(ldexpf(g[j], grow));
                *reinterpret_cast<u32x4 *>(a.gh + at * 32 * DT + col) = __builtin_bit_cast(u32x4, h);
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = 0.0f;
                if (there) load8_any(a.q.p, b * a.q.sb + where.t * a.q.st + head * a.q.sh + col, count, q, a.codes, a.f);
                *reinterpret_cast<u32x4 *>(a.qh + at * 32 * DT + col) = half_signed(to_half(q, a.up, high_q), s.scale);
            }
        }
        if constexpr (HALF) {
            high_q = block_max(high_q, shared);
            if (threadIdx.x == 0) a.highs[blockIdx.x] = high_q;
        }
    } else if constexpr (HALF) {
        const uint32_t n = blockIdx.x - row_blocks, tile = n % key_packs, bkh = n / key_packs;
        const int kh = static_cast<int>(bkh % s.kv_heads), b = static_cast<int>(bkh / s.kv_heads);
        const AttnSeq seq = attn_seq(s, b);
        uint32_t high_k = 0, high_v = 0;
#pragma unroll 1
        for (int r = in; r < kPackRows; r += kStep) {
            const int key = static_cast<int>(tile) * kPackRows + r;
            const int64_t at = static_cast<int64_t>(bkh) * a.key_tiles * kKvKeys + key;
            float k[8], v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) k[j] = v[j] = 0.0f;
            if (key < seq.length && count > 0) {
                load8_any(a.k.p, b * a.k.sb + key * a.k.st + kh * a.k.sh + col, count, k, a.codes, a.f);
                load8_any(a.v.p, b * a.v.sb + key * a.v.st + kh * a.v.sh + col, count, v, a.codes, a.f);
            }
            *reinterpret_cast<u32x4 *>(a.kh + at * 32 * DT + col) = to_half(k, a.up, high_k);
            *reinterpret_cast<u32x4 *>(a.vh + at * 32 * DT + col) = to_half(v, a.up, high_v);
        }
        high_k = block_max(high_k, shared);
        high_v = block_max(high_v, shared);
        if (threadIdx.x == 0) {
            const uint32_t key_blocks = key_packs * s.kv_heads * s.batch;
            a.highs[row_blocks + n] = high_k;
            a.highs[row_blocks + key_blocks + n] = high_v;
        }
    }
}

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

// Keys whose dK and dV a workgroup adds up over (a part of) the rows that may see them.
struct KeyBlock {
    int b, kh, part, k0, key, rows, first, last;
    bool live, used;
    int64_t info;
    AttnSeq seq;
};
__device__ __forceinline__ KeyBlock key_block(const AttnBwd &a, uint32_t id, int step)
{
    const AttnShape &s = a.s;
    KeyBlock k;
    const uint32_t part = id % a.parts, tile = id / a.parts % a.key_tiles, rest = id / a.parts / a.key_tiles;
    k.kh = static_cast<int>(rest % s.kv_heads);
    k.b = static_cast<int>(rest / s.kv_heads);
    k.part = static_cast<int>(part);
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
    if (t0 < t1) {                       // in tiles of `step` rows, and of these the part
        const int64_t n0 = t0 * s.group / step, n1 = (t1 * s.group + step - 1) / step, n = n1 - n0;
        k.first = static_cast<int>(n0 + n * k.part / a.parts) * step;
        k.last = static_cast<int>(n0 + n * (k.part + 1) / a.parts) * step;
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
    const int64_t whole = static_cast<int64_t>(s.batch) * s.k_len * s.kv_heads * s.dim;
    const int64_t at = ((static_cast<int64_t>(k.b) * s.k_len + k.key) * s.kv_heads + k.kh) * s.dim + k.part * whole;
    const bool part = a.parts > 1;
    void *kout = part ? a.part : const_cast<void *>(a.dk.p), *vout = part ? a.part + a.parts * whole : const_cast<void *>(a.dv.p);
    const int64_t kbase = part ? at : k.b * a.dk.sb + k.key * a.dk.st + k.kh * a.dk.sh;
    const int64_t vbase = part ? at : k.b * a.dv.sb + k.key * a.dv.st + k.kh * a.dv.sh;
    const int result = part ? FMT_RESULT_F32 : a.result;
    store_row<DT>(kout, kbase, half, s.dim, dk, kscale, result, a.f);
    store_row<DT>(vout, vbase, half, s.dim, dv, vscale, result, a.f);
}

// dK and dV from their parts, in order: a thread takes four columns.
__global__ __launch_bounds__(256) void attn_parts_kernel(AttnBwd a)
{
    const AttnShape &s = a.s;
    const int fours = (s.dim + 3) / 4;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, tokens = static_cast<int64_t>(s.batch) * s.k_len * s.kv_heads;
    if (n >= 2 * tokens * fours) return;
    const bool value = n >= tokens * fours;
    const int64_t i = value ? n - tokens * fours : n, token = i / fours, whole = tokens * s.dim;
    const int col = static_cast<int>(i % fours) * 4, count = min(s.dim - col, 4);
    const float *p = a.part + (value ? a.parts * whole : 0) + token * s.dim + col;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int part = 0; part < a.parts; ++part, p += whole)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < count) v[j] += p[j];
    const AttnView &out = value ? a.dv : a.dk;
    const int kh = static_cast<int>(token % s.kv_heads), key = static_cast<int>(token / s.kv_heads % s.k_len), b = static_cast<int>(token / s.kv_heads / s.k_len);
    store4(const_cast<void *>(out.p), b * out.sb + key * out.st + kh * out.sh + col, count, v, a.result, a.f);
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
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const KeyBlock key = key_block(a, id, kKvRows);
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

// Both in one launch, workgroups of keys first: all of them (no flags), or those that the launch before has flagged, among few that stay.
template <int DT>
__global__ __launch_bounds__(256) void attn_bwd_kernel(AttnBwd a)
{
    __shared__ union Shared {
        DqShared<DT> q;
        DkvShared<DT> kv;
        __device__ Shared() {}
    } sh;
    for (uint32_t i = blockIdx.x; i < a.key_blocks + a.row_blocks; i += gridDim.x) {
        const bool keys = i < a.key_blocks;
        const uint32_t id = keys ? xcd_order(i, a.key_blocks) : xcd_order(i - a.key_blocks, a.row_blocks);
        if (a.flags && a.flags[keys ? id : a.key_blocks + id] == 0) continue;        // (the same in the whole workgroup)
        if (keys) dkv_pieces<DT>(a, id, sh.kv);
        else dq_pieces<DT>(a, id, sh.q);
        __syncthreads();
    }
}

// ---- operands of one fp16 value each, P and dS in NP pieces of fp16
//
// A row of dO is taken times its own power of two, 2^grow, which brings its largest element to [2^11, 2^12): dP and dS of a row carry that
// factor.  dQ loses it at the end.  dK and dV add up rows: there P and dS of a row are taken times 2^(c - grow), with c the smallest grow so
// far, and sums are brought along when c falls.  A |dS| that fp16 does not hold flags the workgroup as operands out of range do.

// The largest magnitudes of what a workgroup reads, as bit patterns.
struct Highs {
    uint32_t q = 0, k = 0, v = 0, ds = 0;
};

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
        for (int i = 0; i < count / kPackRows; ++i) h = max(h, p[first / kPackRows + i]);
        return h;
    }
};

__device__ __forceinline__ void half_flags(const AttnBwd &a, uint32_t at, const Highs &h)
{
    bool bad = h.ds > __float_as_uint(65504.0f);
    if (a.check) {                                     // q, k and v are the same in the whole workgroup
        const uint32_t least = __float_as_uint(kHalfLeast);
        bad |= max(max(h.q, h.k), h.v) >= __float_as_uint(kHalfLimit);
        bad |= (h.q != 0u && h.q < least) || (h.k != 0u && h.k < least) || (h.v != 0u && h.v < least);
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) a.flags[at] = bad;
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

template <int DT>
struct DqHalfShared {
    AttnTile<1, DT, kKeyTile> ks[2], vs[2];
};

template <int NP, int DT>
__device__ __forceinline__ void dq_half(const AttnBwd &a, uint32_t id, DqHalfShared<DT> &sh)
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
    for (int n = 0; n < count; ++n) {
        const int tile = tiles.at(n), k0 = tile * kKeyTile, buf = n & 1;
        kr.put(sh.ks[buf]);
        vr.put(sh.vs[buf]);
        high.k = max(high.k, highs.of(highs.k, k0, kKeyTile));
        high.v = max(high.v, highs.of(highs.v, k0, kKeyTile));
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
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float ds[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = exp2_fast(fmaf(x[8 * kb + j], scale2, -lse2));
                    ds[j] = p == 0.0f ? 0.0f : p * fmaf(dp[8 * kb + j], down, -delta);
                    high.ds = max(high.ds, __float_as_uint(ds[j]) & 0x7FFFFFFFu);
                }
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
    half_flags(a, a.key_blocks + id, high);
    store_dq<DT>(a, r, dq, ldexpf(s.scale * down, grow == kNoRow ? 0 : -static_cast<int>(grow)));
}

template <int DT>
constexpr int kHalfRows = DT == 2 ? 64 : 32;

template <int DT>
struct DkvHalfShared {
    AttnTile<1, DT, kHalfRows<DT>> qs[2], gs[2];
    alignas(16) float lse[2][kHalfRows<DT>], delta[2][kHalfRows<DT>], weight[2][kHalfRows<DT>];
    float least[2];
};

template <int NP, int DT>
__device__ __forceinline__ void dkv_half(const AttnBwd &a, uint32_t id, DkvHalfShared<DT> &sh)
{
    constexpr int kRows = kHalfRows<DT>, DP = 32 * DT;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const KeyBlock key = key_block(a, id, kRows);
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
    // rows that see the lane's key
    int seen_from = 0;
    uint32_t seen = 0;
    if (key.used) {
        int64_t t0 = 0, t1 = s.q_len;
        if (s.causal) t0 = max(t0, static_cast<int64_t>(key.key) - key.seq.first);
        if (s.window && key.key >= s.sinks) {
            t0 = max(t0, static_cast<int64_t>(key.key) - s.window + 1 - key.seq.first);
            t1 = min(t1, static_cast<int64_t>(key.key) + s.window - key.seq.first);
        }
        if (t0 < t1) {
            seen_from = static_cast<int>(t0 * s.group);
            seen = static_cast<uint32_t>((t1 - t0) * s.group);
        }
    }
    float least = kNoRow, running = kNoRow;      // the smallest grow: of the sums, and (wave 0) of the rows read so far
    int buf = 0;
    for (int row0 = key.first; row0 < key.last; row0 += kRows, buf ^= 1) {
        qr.put(sh.qs[buf]);
        gr.put(sh.gs[buf]);
        high.q = max(high.q, highs.of(highs.q, row0, kRows));
        if (threadIdx.x < 64) {
            float low = info[2];
#pragma unroll
            for (int w = 32; w > 0; w >>= 1) low = fminf(low, __shfl_xor(low, w));
            running = fminf(running, low);
            if (threadIdx.x < kRows) {
                sh.lse[buf][threadIdx.x] = info[0];
                sh.delta[buf][threadIdx.x] = info[1];
                sh.weight[buf][threadIdx.x] = info[2] == kNoRow ? 0.0f : ldexpf(1.0f, static_cast<int>(running - info[2]));
            }
            if (threadIdx.x == 0) sh.least[buf] = running;
        }
        __syncthreads();
        if (row0 + kRows < key.last) fetch(row0 + kRows);
        const float next = sh.least[buf];
        if (next < least) {                                        // the same in the whole workgroup
            const float bring = least == kNoRow ? 1.0f : ldexpf(1.0f, static_cast<int>(next - least));
            least = next;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    dk[d][i] *= bring;
                    dv[d][i] *= bring;
                }
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
                    x[i] = static_cast<uint32_t>(row0 + 32 * rt + 8 * (i / 4) + 4 * half + (i & 3) - seen_from) < seen ? x[i] : -INFINITY;
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float p[8], ds[8];
#pragma unroll
                for (int j0 = 0; j0 < 8; j0 += 4) {
                    const int row = 32 * rt + 16 * kb + 2 * j0 + 4 * half;
                    const f32x4 lse = *reinterpret_cast<const f32x4 *>(&sh.lse[buf][row]), delta = *reinterpret_cast<const f32x4 *>(&sh.delta[buf][row]);
                    const f32x4 weight = *reinterpret_cast<const f32x4 *>(&sh.weight[buf][row]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = exp2_fast(fmaf(x[8 * kb + j0 + j], scale2, -lse[j])) * weight[j];
                        const float d = e == 0.0f ? 0.0f : e * fmaf(dp[8 * kb + j0 + j], down, -delta[j]);
                        p[j0 + j] = e * 16384.0f;
                        ds[j0 + j] = d;
                        high.ds = max(high.ds, __float_as_uint(d) & 0x7FFFFFFFu);
                    }
                }
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
    half_flags(a, id, high);
    const int lose = least == kNoRow ? 0 : -static_cast<int>(least);
    store_dkv<DT>(a, key, dk, dv, ldexpf(fabsf(s.scale) * down, lose), ldexpf(1.0f / 16384.0f, lose));
}

template <int NP, int DT>
__global__ __launch_bounds__(256, DT == 2 ? 2 : 1) void attn_bwd_half_kernel(AttnBwd a)
{
    __shared__ union Shared {
        DqHalfShared<DT> q;
        DkvHalfShared<DT> kv;
        __device__ Shared() {}
    } sh;
    if (blockIdx.x < a.key_blocks) dkv_half<NP, DT>(a, xcd_order(blockIdx.x, a.key_blocks), sh.kv);
    else dq_half<NP, DT>(a, xcd_order(blockIdx.x - a.key_blocks, a.row_blocks), sh.q);
}

}  // namespace

int launch_attention_bwd(const AttnShape &s, const AttnView &q, const AttnView &k, const AttnView &v, const AttnView &o, const AttnView &go,
                         const float *lse, const AttnView &dq, const AttnView &dk, const AttnView &dv, int32_t store, int32_t result,
                         const ElemFormat &f, fmt_format_t fmt, hipStream_t stream)
{
    AttnBwd a{};
    a.s = s;
    a.q = q, a.k = k, a.v = v, a.o = o, a.go = go, a.dq = dq, a.dk = dk, a.dv = dv;
    a.lse = lse;
    a.result = result;
    a.f = f;
    int cus = 0;
    int rc = device_cu_count(&cus);
    if (rc != FMT_OK) return rc;
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, rows = static_cast<int64_t>(s.q_len) * s.group;
    if (all_rows == 0) a.s.q_len = 0;            // no queries: dK and dV are zero
    a.row_tiles = static_cast<uint32_t>(all_rows == 0 ? 0 : (rows + kRowTile - 1) / kRowTile);
    a.key_tiles = static_cast<uint32_t>((s.k_len + kKvKeys - 1) / kKvKeys);
    // few keys, many rows: their rows in parts of 256 or more, until the compute units have two workgroups each
    const int64_t blocks = static_cast<int64_t>(a.key_tiles) * s.kv_heads * s.batch;
    int64_t parts = blocks == 0 ? 1 : std::min((2 * cus + blocks - 1) / blocks, rows / 256);
    a.parts = static_cast<int32_t>(std::max<int64_t>(parts, 1));
    const int64_t key_blocks = blocks * a.parts, row_blocks = static_cast<int64_t>(a.row_tiles) * s.kv_heads * s.batch;
    if (key_blocks + row_blocks > 0x1FFFFFFF) return FMT_ERR_SHAPE;
    a.key_blocks = static_cast<uint32_t>(key_blocks);
    a.row_blocks = static_cast<uint32_t>(row_blocks);
    if (key_blocks + row_blocks == 0) return FMT_OK;
    const bool half = attention_half(fmt);
    a.codes = store == FMT_STORE_CODE16;
    a.gcodes = result == FMT_RESULT_CODE16;
    a.check = fmt.e > 5;
    a.up = a.check ? kHalfUp : 1.0f;

    // scratch: fp16 operands first (rows of 64 or 128 bytes), then words
    const int64_t bkh = static_cast<int64_t>(s.batch) * s.kv_heads, width = s.dim <= 64 ? 64 : 128;
    const int64_t prows = bkh * a.row_tiles * kRowTile, pkeys = bkh * a.key_tiles * kKvKeys, whole = static_cast<int64_t>(s.batch) * s.k_len * s.kv_heads * s.dim;
    static_assert(kRowTile / kPackRows == 4 && kKvKeys / kPackRows == 4);
    const int64_t operands = half ? (prows + pkeys) * width : 0, nhighs = half ? 4 * bkh * (a.row_tiles + 2 * a.key_tiles) : 0;      // words: two tensors of half a word
    const int64_t nflags = half ? key_blocks + row_blocks : 0, nparts = a.parts > 1 ? 2 * a.parts * whole : 0;
    float *scratch = nullptr;
    rc = get_acc_scratch(stream, static_cast<size_t>(operands + 4 * prows + nhighs + nflags + nparts + 1) * sizeof(float), &scratch);
    if (rc != FMT_OK) return rc;
    if (half) {
        a.qh = reinterpret_cast<uint16_t *>(scratch);
        a.gh = a.qh + prows * width;
        a.kh = a.gh + prows * width;
        a.vh = a.kh + pkeys * width;
        a.highs = reinterpret_cast<uint32_t *>(scratch + operands + 4 * prows);
        a.flags = a.highs + nhighs;
    }
    a.info = scratch + operands;
    a.part = scratch + operands + 4 * prows + nhighs + nflags;

    const dim3 threads(256);
    const uint32_t blocks_all = a.key_blocks + a.row_blocks, tiles = 4 * static_cast<uint32_t>(bkh) * (a.row_tiles + (half ? a.key_tiles : 0));
    with_dim(s.dim, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (tiles && half) attn_pack_kernel<DT, true><<<dim3(tiles), threads, 0, stream>>>(a);
        else if (tiles) attn_pack_kernel<DT, false><<<dim3(tiles), threads, 0, stream>>>(a);
        if (half && half_pieces(fmt, result) == 2) attn_bwd_half_kernel<2, DT><<<dim3(blocks_all), threads, 0, stream>>>(a);
        else if (half) attn_bwd_half_kernel<1, DT><<<dim3(blocks_all), threads, 0, stream>>>(a);
        attn_bwd_kernel<DT><<<dim3(half ? std::min(blocks_all, static_cast<uint32_t>(cus)) : blocks_all), threads, 0, stream>>>(a);
    });
    if (a.parts > 1) {
        const int64_t n = 2 * whole / s.dim * ((s.dim + 3) / 4);
        attn_parts_kernel<<<dim3(static_cast<uint32_t>((n + 255) / 256)), threads, 0, stream>>>(a);
    }
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
