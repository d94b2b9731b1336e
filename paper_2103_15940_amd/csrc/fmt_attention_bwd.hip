// Attention, backward: what runs before and after the products, and the choice of kernels.
#include <algorithm>

#include "fmt_attention_bwd.h"

namespace fmt {

extern template void run_attention_bwd<2>(const AttnBwd &, bool, bool, dim3, hipStream_t);
extern template void run_attention_bwd<4>(const AttnBwd &, bool, bool, dim3, hipStream_t);

namespace {

// join over a workgroup, of magnitudes and what else there is to know (most often nothing).
__device__ __forceinline__ uint32_t block_join(uint32_t high, uint32_t more, uint32_t *shared)
{
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) high = max(high, static_cast<uint32_t>(__shfl_xor(static_cast<int>(high), w)));
    high &= 0x7FFFFF00u;
    if (__builtin_expect(__any(more != 0u), 0)) {
#pragma unroll
        for (int w = 32; w > 0; w >>= 1) more = join(more, static_cast<uint32_t>(__shfl_xor(static_cast<int>(more), w)));
        high |= more;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = high;
    __syncthreads();
    return join(join(shared[0], shared[1]), join(shared[2], shared[3]));
}

// Whether one of eight values, as they go to fp16, may lose bits.
__device__ __forceinline__ bool may_cut(const float (&v)[8], float up, float whole)
{
    uint32_t low = 0xFFFFFFFFu;
#pragma unroll
    for (int j = 0; j < 8; j += 2) low = min(min((__float_as_uint(v[j] * up) << 1) - 1u, (__float_as_uint(v[j + 1] * up) << 1) - 1u), low);
    return low < (__float_as_uint(whole) << 1) - 1u;
}

// How many of eight values in fp16 are not zero.
__device__ __forceinline__ int count_of(const u32x4 &h)
{
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += ((h[i] & 0x7FFFu) != 0u) + ((h[i] & 0x7FFF0000u) != 0u);
    return n;
}

// Over the lanes of a row.
template <int LANES>
__device__ __forceinline__ int lanes_total(int n)
{
#pragma unroll
    for (int w = LANES / 2; w > 0; w >>= 1) n += __shfl_xor(n, w);
    return n;
}

// What the products need: of 32 rows delta = sum over the head's columns of R(dO) O, lse, and with HALF R(Q) and R(dO) as fp16 operands; with HALF
// also of 32 keys R(K) and R(V).  4 DT lanes per row, 8 columns each.  One pass over the tensors, whose tiles are then read many times.
// (42 MB read and 34 written for 4 x 1024 tokens with 16 heads of 64, 16 us: 4096 workgroups of one pass each.)
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
        uint32_t high_q = 0, more = 0;
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
            const int grow = min(max(141 - static_cast<int>(high >> 23), -120), 120);      // 14 - the exponent of the largest
            float q[8], scaled[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] = 0.0f;
                scaled[j] = ldexpf(g[j], grow);
            }
            bool lost = false;
            if constexpr (HALF) {
                if (there) load8_any(a.q.p, b * a.q.sb + where.t * a.q.st + head * a.q.sh + col, count, q, a.codes, a.f);
                *reinterpret_cast<u32x4 *>(a.qh + at * 32 * DT + col) = half_signed(to_half(q, a.up, high_q), s.scale);
                uint32_t ignore = 0;
                *reinterpret_cast<u32x4 *>(a.gh + at * 32 * DT + col) = to_half(scaled, 1.0f, ignore);
                if (__builtin_expect(__any(may_cut(scaled, 1.0f, a.whole) || may_cut(q, a.up, a.whole)), 0)) {
                    bool q_lost = false;
                    const int cut_q = count_of(half_rest(q, a.up, q_lost)), cut_g = lanes_total<kEights>(count_of(half_rest(scaled, 1.0f, lost)));
                    lost = lanes_total<kEights>(lost) != 0;
                    if (q_lost) high_q = 0x7F800000u;
                    more = join(more, static_cast<uint32_t>(cut_g) | (cut_q + cut_g ? 0x80000000u : 0u));
                }
            }
            if (col == 0) {
                const float lse = row < rows ? a.lse[(static_cast<int64_t>(b) * s.heads + head) * s.q_len + where.t] : -INFINITY;
                a.info[kInfoLse2 * all + at] = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
                a.info[kInfoDelta * all + at] = sum;
                a.info[kInfoGrow * all + at] = high == 0u ? kNoRow : static_cast<float>(grow);
                // (an infinity or NaN in dO, or bits of it that not even a second fp16 value holds, make NaN of the row, and so of the check on dS)
                a.info[kInfoScaledDelta * all + at] = high >= 0x7F800000u || lost ? NAN : ldexpf(sum, grow);
            }
        }
        if constexpr (HALF) {
            high_q = block_join(high_q, more, shared);
            if (threadIdx.x == 0) a.highs[blockIdx.x] = high_q;
        }
    } else if constexpr (HALF) {
        const uint32_t n = blockIdx.x - row_blocks, tile = n % key_packs, bkh = n / key_packs;
        const int kh = static_cast<int>(bkh % s.kv_heads), b = static_cast<int>(bkh / s.kv_heads);
        const AttnSeq seq = attn_seq(s, b);
        uint32_t high_k = 0, high_v = 0, more_k = 0, more_v = 0;
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
            if (__builtin_expect(__any(may_cut(k, a.up, a.whole) || may_cut(v, a.up, a.whole)), 0)) {
                bool k_lost = false, ignore = false;
                if (count_of(half_rest(k, a.up, k_lost))) more_k = 0x80000000u;
                if (k_lost) high_k = 0x7F800000u;
                more_v = join(more_v, static_cast<uint32_t>(lanes_total<kEights>(count_of(half_rest(v, a.up, ignore)))));
            }
        }
        high_k = block_join(high_k, more_k, shared);
        high_v = block_join(high_v, more_v, shared);
        if (threadIdx.x == 0) {
            const uint32_t key_blocks = key_packs * s.kv_heads * s.batch;
            a.highs[row_blocks + n] = high_k;
            a.highs[row_blocks + key_blocks + n] = high_v;
        }
    }
}

// dK and dV from their parts, in order: a thread takes four columns (6 us, most of it its launch and one trip to memory).
__global__ __launch_bounds__(256) void attn_parts_kernel(AttnBwd a)
{
    const AttnShape &s = a.s;
    const int fours = (s.dim + 3) / 4;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, tokens = static_cast<int64_t>(s.batch) * a.part_keys * s.kv_heads;
    if (n >= 2 * tokens * fours) return;
    const bool value = n >= tokens * fours;
    const int64_t i = value ? n - tokens * fours : n, token = i / fours, whole = tokens * s.dim;
    const int col = static_cast<int>(i % fours) * 4, count = min(s.dim - col, 4);
    const float *p = a.part + (value ? a.parts * whole : 0) + token * s.dim + col;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int part0 = 0; part0 < a.parts; part0 += 8, p += 8 * whole) {
        f32x4 x[8];                                // eight parts on their way at a time
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = load4(p + i * whole, part0 + i < a.parts ? count : 0);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += x[i][j];
    }
    const AttnView &out = value ? a.dv : a.dk;
    const int kh = static_cast<int>(token % s.kv_heads), key = static_cast<int>(token / s.kv_heads % a.part_keys), b = static_cast<int>(token / s.kv_heads / a.part_keys);
    store4(const_cast<void *>(out.p), b * out.sb + key * out.st + kh * out.sh + col, count, v, a.result, a.f);
}

}  // namespace

constexpr int64_t kMostWords = (int64_t)1 << 31;      // of scratch for operands, beyond which a call of several sequences goes in two

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
    const int64_t bkh = static_cast<int64_t>(s.batch) * s.kv_heads, blocks = a.key_tiles * bkh;
    int64_t parts = blocks == 0 ? 1 : std::min((2 * cus + blocks - 1) / blocks, rows / 256);
    a.part_tiles = a.key_tiles;
    if (parts <= 1) {
        parts = 1;
        a.part_tiles = 0;
        // tiles with sinks, which all rows see, where the others are seen from a window: in parts of about as many rows (4 x 1024 tokens with a
        // window of 256: the kernel 78 -> 67 us)
        const int64_t near = (static_cast<int64_t>(s.window) + kKvKeys) * s.group;
        if (s.window > 0 && s.sinks > 0 && rows > 0 && rows >= 2 * near) {      // (no heads: near is 0)
            parts = std::min(rows / near, rows / 256);
            a.part_tiles = std::min(a.key_tiles, static_cast<uint32_t>((std::min(s.sinks, s.k_len) + kKvKeys - 1) / kKvKeys));
            if (parts <= 1) parts = 1, a.part_tiles = 0;
        }
    }
    a.parts = static_cast<int32_t>(parts);
    a.part_keys = static_cast<int32_t>(std::min<int64_t>(s.k_len, static_cast<int64_t>(a.part_tiles) * kKvKeys));
    const int64_t key_blocks = (a.part_tiles * parts + a.key_tiles - a.part_tiles) * bkh, row_blocks = static_cast<int64_t>(a.row_tiles) * s.kv_heads * s.batch;
    const bool half = attention_half(fmt, s);
    const int64_t width = s.dim <= 64 ? 64 : 128;
    const int64_t prows = bkh * a.row_tiles * kRowTile, pkeys = bkh * a.key_tiles * kKvKeys, whole = static_cast<int64_t>(s.batch) * a.part_keys * s.kv_heads * s.dim;
    const int64_t operands = half ? (prows + pkeys) * width : 0;       // words: two tensors of half a word
    const bool too_many = std::max(key_blocks + row_blocks, 4 * bkh * (a.row_tiles + a.key_tiles)) > most_workgroups(256) ||
                          (parts > 1 && 2 * whole > most_workgroups(1));
    if (too_many || operands + 4 * prows > kMostWords) {
        // in two calls, if there are two sequences
        if (s.batch > 1) {
            const int32_t first = s.batch / 2;
            const int64_t in = store == FMT_STORE_CODE16 ? 2 : 4, out = result == FMT_RESULT_CODE16 ? 2 : 4;
            rc = launch_attention_bwd(attn_from(s, 0, first), q, k, v, o, go, lse, dq, dk, dv, store, result, f, fmt, stream);
            if (rc != FMT_OK) return rc;
            return launch_attention_bwd(attn_from(s, first, s.batch - first), attn_from(q, first, in), attn_from(k, first, in), attn_from(v, first, in),
                                        attn_from(o, first, out), attn_from(go, first, out), lse + static_cast<int64_t>(first) * s.heads * s.q_len,
                                        attn_from(dq, first, out), attn_from(dk, first, out), attn_from(dv, first, out), store, result, f, fmt, stream);
        }
        if (too_many) return FMT_ERR_SHAPE;
    }
    a.key_blocks = static_cast<uint32_t>(key_blocks);
    a.row_blocks = static_cast<uint32_t>(row_blocks);
    if (key_blocks + row_blocks == 0) return FMT_OK;
    a.codes = store == FMT_STORE_CODE16;
    a.gcodes = result == FMT_RESULT_CODE16;
    a.check = fmt.e > 5;
    a.up = a.check ? kHalfUp : 1.0f;
    a.whole = ldexpf(1.0f, fmt.m - 24);
    a.limit = a.check && half ? ldexpf(1.0f, score_limit(s)) : 0.0f;

    // scratch: fp16 operands first (rows of 64 or 128 bytes), then words
    static_assert(kRowTile / kPackRows == 4 && kKvKeys / kPackRows == 4);
    const int64_t nhighs = half ? 4 * bkh * (a.row_tiles + 2 * a.key_tiles) : 0;
    const int64_t nparts = a.parts > 1 ? 2 * a.parts * whole : 0;
    float *scratch = nullptr;
    rc = get_acc_scratch(stream, static_cast<size_t>(operands + 4 * prows + nhighs + nparts + 1) * sizeof(float), &scratch);
    if (rc != FMT_OK) return rc;
    if (half) {
        a.qh = reinterpret_cast<uint16_t *>(scratch);
        a.gh = a.qh + prows * width;
        a.kh = a.gh + prows * width;
        a.vh = a.kh + pkeys * width;
        a.highs = reinterpret_cast<uint32_t *>(scratch + operands + 4 * prows);
    }
    a.info = scratch + operands;
    a.part = scratch + operands + 4 * prows + nhighs;

    const dim3 threads(256);
    const uint32_t blocks_all = a.key_blocks + a.row_blocks, tiles = 4 * static_cast<uint32_t>(bkh) * (a.row_tiles + (half ? a.key_tiles : 0));
    with_dim(s.dim, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (tiles && half) attn_pack_kernel<DT, true><<<dim3(tiles), threads, 0, stream>>>(a);
        else if (tiles) attn_pack_kernel<DT, false><<<dim3(tiles), threads, 0, stream>>>(a);
    });
    if (s.dim <= 64) run_attention_bwd<2>(a, half, half_pieces(fmt, result) == 2, dim3(blocks_all), stream);
    else run_attention_bwd<4>(a, half, half_pieces(fmt, result) == 2, dim3(blocks_all), stream);
    if (a.parts > 1) {
        const int64_t n = 2 * whole / s.dim * ((s.dim + 3) / 4);
        attn_parts_kernel<<<dim3(static_cast<uint32_t>((n + 255) / 256)), threads, 0, stream>>>(a);
    }
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
