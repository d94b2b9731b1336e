// Attention on the matrix cores: what its kernels share.
//
//   S = scale R(Q) R(K)^T, visible pairs only;  P = exp(S - lse), lse = log sum exp S of a row;  O = P R(V)
//   delta = sum R(dO) O;  dP = R(dO) R(V)^T;  dS = P (dP - delta);
//   dQ = scale dS R(K);  dK = scale dS^T R(Q);  dV = P^T R(dO)
//
// Key j is visible to the query at position i where j < length, j <= i (causal), and |i - j| < window or j < sinks (window > 0).
//
// Heads that share keys and values are taken as rows of one product: row r is query r / group of head r % group of the group, so a
// tile of keys is read once for all of them, and gradients of shared keys and values add up in the accumulators.
//
// Operands go as one fp16 value each where their range allows, P and dS in one or two fp16 pieces (below).  Otherwise they go in two bf16
// pieces (up to 16 significant bits, fp32's range), whose products are exact in the matrix cores and added in fp32, and P and dS in
// three, which hold all of their 24 bits; products of pieces that lie below 2^-24 of the largest are left out.
//
// Layout of v_mfma_f32_32x32x16: A gives lane l row l % 32 and the 8 k from 8 (l / 32); B the same with columns; the result gives lane l column
// l % 32, and its register i row 8 (i / 4) + 4 (l / 32) + i % 4.  So registers 8b to 8b + 7 of a result are, as they stand, a B operand for
// the 16 k from 16b, in an order of k that its A operand has to follow: the lower lanes have k 0-3 and 8-11, the upper 4-7 and 12-15.  P and
// dS thus go from one product into the next without leaving their lanes; the A operand with that order, and transposed, comes out of LDS
// with ds_read_b64_tr_b16 (16 lanes read 4 rows x 16 columns, lane i receives column i).
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "fmt_elem.h"

namespace fmt {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct AttnSeq {              // one sequence's length and the position of its first query
    int length, first;
};

__device__ __forceinline__ AttnSeq attn_seq(const AttnShape &s, int b)
{
    int length = s.k_len, first = s.k_len - s.q_len;
    if (s.k_lens) length = min(max(s.k_lens[b], 0), s.k_len);
    if (s.q_pos) first = min(max(s.q_pos[b], -(1 << 30)), 1 << 30);
    return AttnSeq{length, first};
}

// Whether key j < length is visible from position i.
__device__ __forceinline__ bool attn_sees(const AttnShape &s, int length, int i, int j)
{
    const int d = i - j;
    const bool near = s.window == 0 || (d < s.window && d > -s.window) || j < s.sinks;
    return j < length && (!s.causal || d >= 0) && near;
}

// The keys that one position sees: [first, first + count) and [0, sinks).
struct AttnKeys {
    int first, sinks;
    uint32_t count;
};
__device__ __forceinline__ AttnKeys attn_keys(const AttnShape &s, int length, int i)
{
    int64_t end = length, begin = 0, sinks = 0;
    if (s.causal) end = min(end, static_cast<int64_t>(i) + 1);
    if (s.window) {
        sinks = min(static_cast<int64_t>(s.sinks), end);
        begin = max(static_cast<int64_t>(0), static_cast<int64_t>(i) - s.window + 1);
        end = min(end, static_cast<int64_t>(i) + s.window);
    }
    return AttnKeys{static_cast<int>(begin < end ? begin : 0), static_cast<int>(sinks), static_cast<uint32_t>(begin < end ? end - begin : 0)};
}

// Scores of keys k0, k0 + 1, ... (register i of a tile's 32 keys holds key 8 (i / 4) + i % 4 from k0) that the lane's position does not see: -inf.
__device__ __forceinline__ void attn_hide(const AttnKeys &m, int k0, f32x16 &x)
{
    const int from = k0 - m.first;
    if (__any(k0 < m.sinks)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int c = 8 * (i / 4) + (i & 3);
            x[i] = static_cast<uint32_t>(from + c) < m.count || k0 + c < m.sinks ? x[i] : -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = static_cast<uint32_t>(from + 8 * (i / 4) + (i & 3)) < m.count ? x[i] : -INFINITY;
    }
}

// Whether every key of [k0, k1) is visible from every position of [i0, i1].
__device__ __forceinline__ bool attn_sees_all(const AttnShape &s, int length, int64_t i0, int64_t i1, int k0, int k1)
{
    const bool near = s.window == 0 || k1 <= s.sinks || (i1 - k0 < s.window && k1 - 1 - i0 < s.window);
    return k1 <= length && (!s.causal || k1 - 1 <= i0) && near;
}

// Keys that positions [i0, i1] may see: tiles of `tile` keys, [0, sinks) and [first, last).
struct AttnTiles {
    int sinks, first, last;
    __device__ int count() const { return sinks + max(0, last - first); }
    __device__ int at(int n) const { return n < sinks ? n : first + (n - sinks); }
};

__device__ __forceinline__ AttnTiles attn_tiles(const AttnShape &s, int length, int64_t i0, int64_t i1, int tile)
{
    int64_t end = length, begin = 0, sinks = 0;
    if (s.causal) end = min(end, i1 + 1);
    if (s.window) {
        sinks = min(static_cast<int64_t>(s.sinks), end);
        begin = max(static_cast<int64_t>(0), i0 - s.window + 1);
        end = min(end, i1 + s.window);
    }
    AttnTiles t;
    t.sinks = sinks > 0 ? static_cast<int>((sinks + tile - 1) / tile) : 0;
    t.first = max(static_cast<int>(min(begin, static_cast<int64_t>(length)) / tile), t.sinks);
    t.last = end > 0 ? static_cast<int>((end + tile - 1) / tile) : 0;
    return t;
}

// The upper halves of two fp32 patterns in one register.
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// Eight fp32 values as N bf16 pieces whose sum they are (N == 1: to nearest; a last piece that cannot hold the rest: to nearest).
template <int N>
__device__ __forceinline__ void bf16_pieces(const float (&v)[8], u32x4 (&out)[N])
{
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n == N - 1) {
            bf16x8 last;
#pragma unroll
            for (int i = 0; i < 8; ++i) last[i] = static_cast<__bf16>(rest[i]);
            out[n] = __builtin_bit_cast(u32x4, last);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t a = __float_as_uint(rest[i]), b = __float_as_uint(rest[i + 1]);
                out[n][i / 2] = upper_halves(a, b);
                rest[i] = __fsub_rn(rest[i], __uint_as_float(a & 0xFFFF0000u));
                rest[i + 1] = __fsub_rn(rest[i + 1], __uint_as_float(b & 0xFFFF0000u));
            }
        }
    }
}

__device__ __forceinline__ f32x16 mfma_bf16(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// acc += A B over all pairs of pieces that count: NA + NB - 2 is the last order that three pieces of one side leave (24 bits).
template <int NA, int NB>
__device__ __forceinline__ f32x16 mfma_pieces(const u32x4 (&a)[NA], const u32x4 (&b)[NB], f32x16 acc)
{
    constexpr int kMost = NA > 2 || NB > 2 ? 2 : NA + NB;
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)
#pragma unroll
        for (int j = NB - 1; j >= 0; --j)
            if (i + j <= kMost) acc = mfma_bf16(a[i], b[j], acc);
    return acc;
}

// Tiles in LDS: [piece][row][columns and padding].  Row reads take 16 bytes of neighbouring rows, column reads 32 bytes of four: at
// a pitch of 36 or 72 dwords neither meets in a bank (32 or 64 dwords, and 68: measured 1.2 to 1.7 times as long).
template <int DT>
constexpr int kAttnPitch = DT == 2 ? 72 : 144;

template <int NQ, int DT, int ROWS>
struct alignas(16) AttnTile {
    uint16_t e[NQ][ROWS][kAttnPitch<DT>];
};

// A (or B) operand: row `row`, 8 columns from `col`.
template <int NQ, int DT, int ROWS>
__device__ __forceinline__ void read_rows(const AttnTile<NQ, DT, ROWS> &t, int row, int col, u32x4 (&out)[NQ])
{
#pragma unroll
    for (int n = 0; n < NQ; ++n) out[n] = *reinterpret_cast<const u32x4 *>(&t.e[n][row][col]);
}

__device__ __forceinline__ s16x4 read_transposed4(const uint16_t *p)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
}

// A operand of the transposed tile: its 32 columns from `col` as rows, its 16 rows from `row` as k, in the order of a result's registers.
template <int NQ, int DT, int ROWS>
__device__ __forceinline__ void read_columns(const AttnTile<NQ, DT, ROWS> &t, int row, int col, int lane, u32x4 (&out)[NQ])
{
    const int r = row + 4 * (lane >> 5) + ((lane & 15) >> 2), c = col + (lane & 16) + 4 * (lane & 3);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const s16x4 lo = read_transposed4(&t.e[n][r][c]), hi = read_transposed4(&t.e[n][r + 8][c]);
        s16x8 both;
#pragma unroll
        for (int i = 0; i < 4; ++i) both[i] = lo[i], both[4 + i] = hi[i];
        out[n] = __builtin_bit_cast(u32x4, both);
    }
}

// Tokens [first, first + ROWS) of one head (of which those before `end` exist) into a tile.
template <int NQ, int DT, int ROWS>
__device__ __forceinline__ void load_tokens(AttnTile<NQ, DT, ROWS> &t, const void *x, int64_t base, int64_t stride, int first, int end, int dim,
                                            bool codes, const ElemFormat &f)
{
    constexpr int kEights = 4 * DT;
#pragma unroll 1
    for (int i = 0; i < ROWS * kEights / 256; ++i) {
        const int n = threadIdx.x + 256 * i, row = n / kEights, col = (n % kEights) * 8;
        const int count = first + row < end ? min(dim - col, 8) : 0;
        float v[8];
        if (count > 0) {
            load8_any(x, base + (first + row) * stride + col, count, v, codes, f);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        }
        u32x4 p[NQ];
        bf16_pieces<NQ>(v, p);
#pragma unroll
        for (int k = 0; k < NQ; ++k) *reinterpret_cast<u32x4 *>(&t.e[k][row][col]) = p[k];
    }
}

// ---- operands as one fp16 value each
//
// Formats of at most 10 stored mantissa bits fit fp16's significand, and 1/5/10 and narrower its range as well: their products are exact in
// one product instead of four of bf16 pieces.  For wider ranges (1/6/9, 1/8/7) values are taken times 2^9, which holds |x| < 2^7 and
// their bits down to 2^-33; what is below is cut.  That puts up to dim 2^-33 (max |Q| + max |K|) |scale| into a score, which is kept to 2^-21 by a limit of Q and K
// (2^7 at most; with a scale of dim^-0.5 it is that).  Where an operand's elements enter a sum of their own channel the cut bits count, whatever other
// channels and tokens hold: a tile with such elements is taken in two parts, and the second, what was cut, times 2^24 more.  A workgroup that meets a larger element,
// an infinity or NaN, or bits below 2^-57, computes its results again with pieces of bf16.  (A second launch
// for such workgroups, which all but a few calls do not have, cost every call 4 us.)
constexpr int kHalfLimit = 7;             // as an exponent
constexpr float kHalfUp = 512.0f, kRestUp = 0x1p24f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mfma_f16(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Eight fp32 values as N fp16 pieces: 11 bits, to nearest, or 22, the first of them cut (its rest goes into the second, to nearest).
template <int N>
__device__ __forceinline__ void f16_pieces(const float (&v)[8], u32x4 (&out)[N])
{
    if constexpr (N == 1) {
        f16x8 h;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = static_cast<_Float16>(v[i]);
        out[0] = __builtin_bit_cast(u32x4, h);
    } else {
        f16x8 lo;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const auto hi = __builtin_amdgcn_cvt_pkrtz(v[i], v[i + 1]);
            out[0][i / 2] = __builtin_bit_cast(uint32_t, hi);
            lo[i] = static_cast<_Float16>(__fsub_rn(v[i], static_cast<float>(hi[0])));
            lo[i + 1] = static_cast<_Float16>(__fsub_rn(v[i + 1], static_cast<float>(hi[1])));
        }
        out[1] = __builtin_bit_cast(u32x4, lo);
    }
}

// Their values in fp32, rounded to the format.
template <bool CODES>
__device__ __forceinline__ void raw_values(const RawEight<CODES> &r, float (&v)[8], const ElemFormat &f)
{
    if constexpr (CODES) {
        uint16_t c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = static_cast<uint16_t>(r.w[0][i / 2] >> (16 * (i & 1)));
        decode_values(c, v, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i / 4][i % 4]);
        round_values(v, f);
    }
}

// fp32 values as fp16 times `up` (their bits fit; what lies below 2^-24 is cut).  high: the largest |x| so far as a bit pattern (NaN above all).
__device__ __forceinline__ u32x4 to_half(const float (&v)[8], float up, uint32_t &high)
{
    u32x4 h;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        high = max(max(__float_as_uint(v[i]) & 0x7FFFFFFFu, __float_as_uint(v[i + 1]) & 0x7FFFFFFFu), high);
        h[i / 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(v[i] * up, v[i + 1] * up));
    }
    return h;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// What codes need on their way to fp16, two at a time: masks of their magnitudes and signs, and for e == 6 the shifts that make fp16
// of them (times 2^9: the exponent field falls by 7).
struct HalfCodes {
    uint32_t body, sign;
    uint32_t scores, limit;                 // limits of Q and K, and of V: as codes, or patterns of unrounded fp32
    uint32_t cut;                           // least magnitude whose bits all fit, as a code less one, or a pattern of fp32, doubled and less one
    int32_t shift, sign_shift;              // shift < 0: by way of fp32
};

// How elements become fp16, known at compile time (elem_kind's ways of rounding, and codes by their format).
enum : int {
    kHalfCodes = 0,      // codes of 1/5/10: as they are
    kHalfFloat = 1,      // fp32, 1/5/10 with denormals: converted
    kBf16Codes = 2,      // codes of 1/8/7
    kSixCodes = 3,       // codes with e == 6, two at a time
    kOtherCodes = 4,     // by way of fp32
    kMagicFloat = 5,     // fp32, e < 8
    kIntegerFloat = 6    // fp32, e == 8
};
constexpr bool half_is_codes(int kind) { return kind == kHalfCodes || kind == kBf16Codes || kind == kSixCodes || kind == kOtherCodes; }
constexpr bool half_has_limit(int kind) { return kind != kHalfCodes && kind != kHalfFloat; }      // e <= 5 otherwise is told at run time

inline int half_kind(fmt_format_t f, int32_t store)
{
    if (store == FMT_STORE_CODE16) return f.e == 5 && f.m == 10 ? kHalfCodes : f.e == 8 && f.m == 7 ? kBf16Codes : f.e == 6 ? kSixCodes : kOtherCodes;
    return f.e == 5 && f.m == 10 && f.denorm ? kHalfFloat : f.e == 8 ? kIntegerFloat : kMagicFloat;
}

// What to_half and raw_half cut off eight values, as fp16 times 2^24 more; lost: what this cuts off too.
__device__ __forceinline__ u32x4 half_rest(const float (&v)[8], float up, bool &lost)
{
    u32x4 h;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const auto top = __builtin_amdgcn_cvt_pkrtz(v[i] * up, v[i + 1] * up);
        const float a = (v[i] * up - static_cast<float>(top[0])) * kRestUp, b = (v[i + 1] * up - static_cast<float>(top[1])) * kRestUp;
        const auto rest = __builtin_amdgcn_cvt_pkrtz(a, b);
        lost |= static_cast<float>(rest[0]) != a || static_cast<float>(rest[1]) != b;
        h[i / 2] = __builtin_bit_cast(uint32_t, rest);
    }
    return h;
}

// Eight elements as fp16 times `up`.  high: the largest magnitude so far; of codes, of either half of a word; of fp32 as a bit pattern, unrounded.
// WATCH: cut tells of elements that may have lost bits.
template <int KIND, bool WATCH>
__device__ __forceinline__ u32x4 raw_half(const RawEight<half_is_codes(KIND)> &r, float up, const HalfCodes &hc, uint32_t &high, bool &cut, const ElemFormat &f)
{
    u32x4 out;
    if constexpr (KIND == kHalfCodes) {
        return r.w[0];
    } else if constexpr (KIND == kHalfFloat) {
        f16x8 h;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = static_cast<_Float16>(__uint_as_float(r.w[i / 4][i % 4]));
        return __builtin_bit_cast(u32x4, h);
    } else if constexpr (KIND == kBf16Codes) {
        u16x2 top = __builtin_bit_cast(u16x2, high), low = {0xFFFF, 0xFFFF};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = r.w[0][i];
            const u16x2 body = __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu);
            top = __builtin_elementwise_max(top, body);
            if constexpr (WATCH) low = __builtin_elementwise_min(low, body - static_cast<uint16_t>(1));
            out[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xFFFF0000u) * up));
        }
        high = __builtin_bit_cast(uint32_t, top);
        if constexpr (WATCH) cut |= min(low[0], low[1]) < hc.cut;
        return out;
    } else if constexpr (KIND == kSixCodes || KIND == kOtherCodes) {
        u16x2 top = __builtin_bit_cast(u16x2, high), low = {0xFFFF, 0xFFFF};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u16x2 body = __builtin_bit_cast(u16x2, r.w[0][i] & hc.body);
            top = __builtin_elementwise_max(top, body);
            low = __builtin_elementwise_min(low, body - static_cast<uint16_t>(1));
        }
        high = __builtin_bit_cast(uint32_t, top);
        if constexpr (KIND == kSixCodes) {
            // a code other than 0 whose fp16 is no normal number (|x| < 2^-23) is rare: then all go by way of fp32
            const uint16_t normal = static_cast<uint16_t>((8u << (10 - hc.shift)) - 1u);
            if (!__any(low[0] < normal || low[1] < normal)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u16x2 body = __builtin_bit_cast(u16x2, r.w[0][i] & hc.body) << static_cast<uint16_t>(hc.shift);
                    const u16x2 h = __builtin_elementwise_sub_sat(body, u16x2{7 << 10, 7 << 10});
                    out[i] = __builtin_bit_cast(uint32_t, h) | (r.w[0][i] & hc.sign) << hc.sign_shift;
                }
                return out;
            }
        }
        float v[8];
        raw_values(r, v, f);
        if constexpr (WATCH) cut |= min(low[0], low[1]) < hc.cut;
        uint32_t ignore = 0;
        return to_half(v, up, ignore);
    } else {
        const QuantParams &p = f.p;
        if constexpr (KIND == kMagicFloat) {
            if (up == 1.0f) {              // e <= 5, no limit: what overflows the format has to become infinity, and NaN stay NaN
                uint32_t u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = r.w[i / 4][i % 4];
                if (__any(run_is_rare(u, p))) {
                    float v[8];
                    raw_values(r, v, f);
                    f16x8 h;
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[i] = static_cast<_Float16>(v[i]);
                    return __builtin_bit_cast(u32x4, h);
                }
            }
        }
        // the short roundings: with a limit, what they do not serve is above it.  (Formats of more than 10 bits do not come here.)
        const uint32_t flush = f.ftz ? p.t_den : 0u;
        const RoundMasks k = round_masks(p);
        auto round = [&](uint32_t u) __attribute__((always_inline)) {
            uint32_t q;
            if constexpr (KIND == kMagicFloat) q = quantize_short<kModeMagic, false, false>(u, p, k);
            else q = (u + p.rbias + __builtin_amdgcn_ubfe(u, p.shift, p.lsb_width)) & p.nmask;
            return __uint_as_float((u & 0x7FFFFFFFu) < flush ? 0u : q);
        };
        uint32_t low = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint32_t a = r.w[i / 4][i % 4], b = r.w[i / 4][i % 4 + 1];
            high = max(max(a & 0x7FFFFFFFu, b & 0x7FFFFFFFu), high);
            const float x = round(a), y = round(b);
            if constexpr (WATCH) low = min(min((__float_as_uint(x) << 1) - 1u, (__float_as_uint(y) << 1) - 1u), low);
            out[i / 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x * up, y * up));
        }
        if constexpr (WATCH) cut |= low < hc.cut;
        return out;
    }
}

// R(Q) is multiplied by the scale's sign, so that scores are ordered as they come out of the product; a scale of 0 makes it 0.
__device__ __forceinline__ u32x4 half_signed(u32x4 q, float scale)
{
    const uint32_t flip = scale < 0.0f ? 0x80008000u : 0u, keep = scale == 0.0f ? 0u : 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = (q[i] ^ flip) & keep;
    return q;
}

// Forward the running maximum stays where it is until a score passes it by 2^4 (a wave of 32 rows would otherwise multiply its sums with some row's factor at
// almost every tile), so P can reach 2^4, and is taken times 2^8: weights keep 22 bits down to 2^-11 of a row's largest, and 11 down to 2^-22.  (The factor comes
// out of the exponential, whose argument has fewer bits the larger it is: with 2^11 ordinary rows' errors were half as large again.)
constexpr float kFwdUp = 8.0f, kFwdSlack = 4.0f;

// Whether a workgroup has to be computed with bf16 pieces: in all of its threads.  Every thread calls it.  high, high_value: what raw_half left.
template <bool CODES>
__device__ __forceinline__ bool half_flag(uint32_t high, uint32_t high_value, const HalfCodes &hc)
{
    const uint32_t h = CODES ? max(high >> 16, high & 0xFFFFu) : high, v = CODES ? max(high_value >> 16, high_value & 0xFFFFu) : high_value;
    return __syncthreads_or(h >= hc.scores || v >= hc.limit);
}

// Workgroups of one launch in an order that gives each of the 8 XCDs (workgroup i runs on XCD i % 8) a run of neighbours, which share keys
// and values in its L2.
__device__ __forceinline__ uint32_t xcd_order(uint32_t i, uint32_t n)
{
    const uint32_t xcd = i & 7, each = n >> 3, more = n & 7;
    return xcd * each + min(xcd, more) + (i >> 3);
}

// 2^x; the vector unit's exponential flushes results below 2^-126, which is below 2^-24 of any sum that holds a 1.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's lse from its largest score in base 2 and the sum of its powers relative to that; -infinity where it sees nothing.
__device__ __forceinline__ float lse_of(float top, float sum) { return sum == 0.0f ? -INFINITY : fmaf(top, 0.6931471805599453f, logf(sum)); }

typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

// A lane's results of DT blocks of 32 columns (its column of the blocks is one row of the tensor): register 4g + i of block d is column
// 32 d + 8 g + 4 half + i, taken times `scale`.  The kind of result is chosen once, ahead of all of them: the paths of the others would
// lie between a wave's stores and cost it misses of the instruction cache (3 us of a call).
template <int DT>
__device__ __forceinline__ void store_row(void *y, int64_t base, int half, int dim, const f32x16 (&o)[DT], float scale, int result, const ElemFormat &f)
{
    auto each = [&](auto put) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * d + 8 * g + 4 * half;
                const float v[4] = {o[d][4 * g] * scale, o[d][4 * g + 1] * scale, o[d][4 * g + 2] * scale, o[d][4 * g + 3] * scale};
                put(col, dim - col, v);
            }
    };
    auto floats = [&](int col, int count, const float (&v)[4]) __attribute__((always_inline)) {
        float *p = static_cast<float *>(y) + base + col;
        if (count >= 4) {
            *reinterpret_cast<f32x4_any *>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) p[i] = v[i];
        }
    };
    auto codes = [&](int col, int count, const uint16_t (&c)[4]) __attribute__((always_inline)) {
        uint16_t *p = static_cast<uint16_t *>(y) + base + col;
        if (count >= 4) {
            *reinterpret_cast<u16x4_any *>(p) = u16x4_any{c[0], c[1], c[2], c[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) p[i] = c[i];
        }
    };
    if (result == FMT_RESULT_F32) {
        each(floats);
    } else if (result == FMT_RESULT_CODE16 && f.codec == kCodecBf16) {
        const float flush = f.ftz ? __uint_as_float(f.p.t_den) : 0.0f;
        each([&](int col, int count, const float (&v)[4]) __attribute__((always_inline)) {
            uint16_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(fabsf(v[i]) < flush ? v[i] * 0.0f : v[i]));
            codes(col, count, c);
        });
    } else if (result == FMT_RESULT_CODE16 && f.codec == kCodecHalf) {
        each([&](int col, int count, const float (&v)[4]) __attribute__((always_inline)) {
            uint16_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = v[i];
                asm("" : "+v"(x));                 // (see round_kind)
                const uint16_t h = __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
                c[i] = v[i] != v[i] ? static_cast<uint16_t>(0x7E00u) : h;
            }
            codes(col, count, c);
        });
    } else {
        each([&](int col, int count, const float (&v)[4]) __attribute__((always_inline)) {
            float r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = v[i];
            round_values(r, f);
            if (result == FMT_RESULT_CODE16) {
                uint16_t c[4];
                encode_values(r, c, f);
                codes(col, count, c);
            } else {
                floats(col, count, r);
            }
        });
    }
}

// Up to four neighbouring values of a part.
__device__ __forceinline__ f32x4 load4(const float *p, int count)
{
    if (count >= 4) return *reinterpret_cast<const f32x4_any *>(p);
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) v[i] = p[i];
    return v;
}

// Up to four neighbouring results of kernels that join parts.
__device__ __forceinline__ void store4(void *y, int64_t at, int count, const float (&v)[4], int result, const ElemFormat &f)
{
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = v[i];
    if (result != FMT_RESULT_F32) round_values(r, f);
    uint16_t c[4];
    if (result == FMT_RESULT_CODE16) encode_values(r, c, f);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) {
            if (result == FMT_RESULT_CODE16) static_cast<uint16_t *>(y)[at + i] = c[i];
            else static_cast<float *>(y)[at + i] = r[i];
        }
}

// run(DT) for a head size.
template <class RUN>
void with_dim(int dim, RUN &&run)
{
    if (dim <= 64) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, 4>{});
}

constexpr int kPieces = 2, kProbPieces = 3;      // bf16 pieces of operands, of P and dS

// Exponent of the limit of Q and K with fp16 operands.
inline int score_limit(const AttnShape &s)
{
    const double most = 2048.0 / (std::fabs(static_cast<double>(s.scale)) * s.dim);
    return most >= 128.0 ? kHalfLimit : std::ilogb(most);
}

// Whether values go as one fp16 value each: the format's fit, and the scale leaves Q and K a limit of 1 or more.
inline bool attention_half(fmt_format_t f, const AttnShape &s) { return f.m <= 10 && (f.e <= 5 || score_limit(s) >= 0); }

inline HalfCodes make_half_codes(fmt_format_t f, const AttnShape &s, int32_t store)
{
    const uint32_t body = (1u << (f.e + f.m)) - 1u, sign = 1u << (f.e + f.m);
    const int bias = (1 << (f.e - 1)) - 1;
    // 2^n; unrounded fp32 is looked at: from 7/8 of it on, what has one mantissa bit becomes 2^n
    auto power = [&](int n) { return store == FMT_STORE_CODE16 ? static_cast<uint32_t>(std::max(bias + n, 0)) << f.m : static_cast<uint32_t>(127 + n) << 23; };
    auto limit = [&](int n) { return power(n) - (store == FMT_STORE_CODE16 ? 0u : 1u << 21); };
    const uint32_t whole = power(f.m - 33), cut = store == FMT_STORE_CODE16 ? (whole ? whole - 1u : 0u) : (whole << 1) - 1u;
    return HalfCodes{body * 0x10001u, sign * 0x10001u, limit(score_limit(s)), limit(kHalfLimit), cut, f.e == 6 ? 10 - f.m : -1, 15 - (f.e + f.m)};
}

// Pieces of P and dS with fp16 operands: one (11 bits) where results have 8, two (22) where they have more.
inline int half_pieces(fmt_format_t f, int32_t result) { return result == FMT_RESULT_F32 || f.m > 7 ? 2 : 1; }

}  // namespace fmt
