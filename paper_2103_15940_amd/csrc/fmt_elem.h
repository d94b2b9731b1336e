// Runs of consecutive elements of the row-wise and attention kernels: fp32 values that are rounded to the format as they are read, or
// the format's own 16-bit codes; and results as unrounded fp32, rounded fp32 or codes.
#pragma once

#include <type_traits>

#include "fmt_quant.h"

namespace fmt {

// Vectors at the alignment of their elements (the memory system takes dword accesses at any address).
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8_any __attribute__((ext_vector_type(8), aligned(2)));

// R of a run; the variant is chosen once for all of it.
template <int N>
__device__ __forceinline__ void round_values(float (&v)[N], const ElemFormat &f)
{
    auto run = [&](auto round) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(round(__float_as_uint(v[i])));
    };
    const QuantParams &p = f.p;
    if (f.codec == kCodecNone) return;
    if (f.codec == kCodecHalf) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            asm("" : "+v"(v[i]));              // (see round_kind)
            v[i] = static_cast<float>(static_cast<_Float16>(v[i]));
        }
        return;
    }
    if (p.mode == kModeInteger) {
        if (f.ftz) run([&](uint32_t u) { return quantize_bits<kModeInteger, true>(u, p); });
        else run([&](uint32_t u) { return quantize_bits<kModeInteger, false>(u, p); });
    } else if (p.mode == kModeMagic) {
        if (f.ftz) run([&](uint32_t u) { return quantize_bits<kModeMagic, true>(u, p); });
        else run([&](uint32_t u) { return quantize_bits<kModeMagic, false>(u, p); });
    } else {
        if (f.ftz) run([&](uint32_t u) { return quantize_bits<kModeMixed, true>(u, p); });
        else run([&](uint32_t u) { return quantize_bits<kModeMixed, false>(u, p); });
    }
}

template <int N>
__device__ __forceinline__ void decode_values(const uint16_t (&c)[N], float (&v)[N], const ElemFormat &f)
{
    if (f.codec == kCodecBf16) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(static_cast<uint32_t>(c[i]) << 16);
    } else if (f.codec == kCodecHalf) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = static_cast<float>(__builtin_bit_cast(_Float16, c[i]));
    } else if (f.p.mode == kModeInteger) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(decode_bits<true>(c[i], f.p));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(decode_bits<false>(c[i], f.p));
    }
}

// Codes of values that are the format's already (round_values' results).
template <int N>
__device__ __forceinline__ void encode_values(const float (&v)[N], uint16_t (&c)[N], const ElemFormat &f)
{
    if (f.codec == kCodecBf16) {
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = static_cast<uint16_t>(__float_as_uint(v[i]) >> 16);
    } else if (f.p.mode == kModeInteger) {
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = static_cast<uint16_t>(encode_bits<kModeInteger>(__float_as_uint(v[i]), f.p));
    } else if (f.codec == kCodecHalf) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint16_t h = __builtin_bit_cast(uint16_t, static_cast<_Float16>(v[i]));
            c[i] = v[i] != v[i] ? static_cast<uint16_t>(0x7E00u) : h;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = static_cast<uint16_t>(encode_bits<kModeMagic>(__float_as_uint(v[i]), f.p));
    }
}

// Eight elements from x[at] on of which the first `count` exist (the others become 0): values of the format in fp32.
template <bool CODES>
__device__ __forceinline__ void load8(const void *x, int64_t at, int count, float (&v)[8], const ElemFormat &f)
{
    if constexpr (CODES) {
        const uint16_t *s = static_cast<const uint16_t *>(x) + at;
        uint16_t c[8];
        if (count >= 8) {
            const u16x8_any w = *reinterpret_cast<const u16x8_any *>(s);
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = i < count ? s[i] : static_cast<uint16_t>(0);
        }
        decode_values(c, v, f);
    } else {
        const float *s = static_cast<const float *>(x) + at;
        if (count >= 8) {
            const f32x4_any a = *reinterpret_cast<const f32x4_any *>(s), b = *reinterpret_cast<const f32x4_any *>(s + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < count ? s[i] : 0.0f;
        }
        round_values(v, f);
    }
}

// The same with the type known at run time (uniform).
__device__ __forceinline__ void load8_any(const void *x, int64_t at, int count, float (&v)[8], bool codes, const ElemFormat &f)
{
    if (codes) load8<true>(x, at, count, v, f);
    else load8<false>(x, at, count, v, f);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight elements as they lie in memory.
template <bool CODES>
struct RawEight {
    u32x4 w[CODES ? 1 : 2];
};

template <bool CODES>
__device__ __forceinline__ RawEight<CODES> raw_load(const void *x, int64_t at, int count)
{
    RawEight<CODES> r;
    typedef std::conditional_t<CODES, u32x4_any2, u32x4_any4> u32x4_any;
#pragma unroll
    for (int n = 0; n < (CODES ? 1 : 2); ++n) r.w[n] = u32x4{0u, 0u, 0u, 0u};
    if (count >= 8) {
        const u32x4_any *s = reinterpret_cast<const u32x4_any *>(static_cast<const char *>(x) + at * (CODES ? 2 : 4));
#pragma unroll
        for (int n = 0; n < (CODES ? 1 : 2); ++n) r.w[n] = s[n];
    } else if (count > 0) {
        if constexpr (CODES) {
            const uint16_t *s = static_cast<const uint16_t *>(x) + at;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) r.w[0][i / 2] |= static_cast<uint32_t>(s[i]) << (16 * (i & 1));
        } else {
            const uint32_t *s = static_cast<const uint32_t *>(x) + at;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) r.w[i / 4][i % 4] = s[i];
        }
    }
    return r;
}

// ---- the same with the way of rounding known at compile time, for kernels that are bound by memory: the paths of other formats would
// lie between their loads and cost them misses of the instruction cache

enum : int {
    kKindNone = 0,     // 1/8/23 with denormals
    kKindHalf = 1,     // 1/5/10 with denormals
    kKindMagic = 2,    // e < 8, m <= 22
    kKindInteger = 3,  // e == 8
    kKindMixed = 4     // e < 8, m == 23
};

inline int elem_kind(const ElemFormat &f)
{
    if (f.codec == kCodecNone) return kKindNone;
    if (f.codec == kCodecHalf) return kKindHalf;
    return f.p.mode == kModeMagic ? kKindMagic : f.p.mode == kModeInteger ? kKindInteger : kKindMixed;
}

// R of eight values.  Where all are below the threshold of infinity (a look of half an instruction each, the same in the whole wave) the short
// forms do; with the flush, e == 8 also asks for values that it would make zero (others than 0, which a dropout leaves many of).
template <int KIND>
__device__ __forceinline__ void round_kind(float (&v)[8], const ElemFormat &f)
{
    if constexpr (KIND == kKindNone) return;
    if constexpr (KIND == kKindHalf) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // the fp32 value itself is what is rounded: product and conversion in one instruction would round once, and lose the sign of -0
            asm("" : "+v"(v[i]));
            v[i] = static_cast<float>(static_cast<_Float16>(v[i]));
        }
    } else {
        const QuantParams &p = f.p;
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(v[i]);
        if constexpr (KIND != kKindMixed) {
            bool rare = run_is_rare(u, p);
            if constexpr (KIND == kKindInteger) {
                if (f.ftz) {
                    uint32_t low = 0xFFFFFFFFu;
#pragma unroll
                    for (int i = 0; i < 8; i += 2) low = min(min((u[i] << 1) - 1u, (u[i + 1] << 1) - 1u), low);
                    rare |= low < (p.t_den << 1) - 1u;
                }
            }
            if (!__any(rare)) {
                if constexpr (KIND == kKindInteger) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((u[i] + p.rbias + __builtin_amdgcn_ubfe(u[i], p.shift, p.lsb_width)) & p.nmask);
                } else {
                    const RoundMasks k = round_masks(p);
                    if (f.ftz) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(quantize_short<kModeMagic, true>(u[i], p, k));
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(quantize_short<kModeMagic, false>(u[i], p, k));
                    }
                }
                return;
            }
        }
        constexpr int kMode = KIND == kKindMagic ? kModeMagic : KIND == kKindInteger ? kModeInteger : kModeMixed;
        const uint32_t flush = f.ftz ? p.t_den : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = quantize_bits<kMode, false>(u[i], p);
            v[i] = __uint_as_float((u[i] & 0x7FFFFFFFu) < flush ? u[i] & 0x80000000u : r);
        }
    }
}

template <int KIND>
__device__ __forceinline__ void decode_kind(const u32x4 &w, float (&v)[8], const ElemFormat &f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = w[i / 2] >> (16 * (i & 1)) & 0xFFFFu;
        if constexpr (KIND == kKindHalf) v[i] = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(c)));
        else if constexpr (KIND == kKindInteger) v[i] = __uint_as_float(c << (31u - f.p.sign_pos));     // the code is the pattern's upper part
        else v[i] = __uint_as_float(decode_bits<false>(c, f.p));
    }
}

// Values of the format to codes.
template <int KIND>
__device__ __forceinline__ u32x4 encode_kind(const float (&v)[8], const ElemFormat &f)
{
    u32x4 w;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        uint32_t c[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float x = v[i + j];
            if constexpr (KIND == kKindHalf) c[j] = __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
            else if constexpr (KIND == kKindInteger) c[j] = __float_as_uint(x) >> (31u - f.p.sign_pos);
            else c[j] = encode_bits<kModeMagic>(__float_as_uint(x), f.p);
        }
        w[i / 2] = c[0] | c[1] << 16;
        if (KIND == kKindHalf) top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(v[i]), fabsf(v[i + 1])), top);
    }
    if constexpr (KIND == kKindHalf) {
        if (__any(top != top)) {                          // any NaN has one code
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] != v[i]) w[i / 2] = (w[i / 2] & (i & 1 ? 0x0000FFFFu : 0xFFFF0000u)) | 0x7E00u << (16 * (i & 1));
        }
    }
    return w;
}

// R of what raw_load gave.
template <int KIND, bool CODES>
__device__ __forceinline__ void kind_values(const RawEight<CODES> &r, float (&v)[8], const ElemFormat &f)
{
    if constexpr (CODES) {
        decode_kind<KIND>(r.w[0], v, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i / 4][i % 4]);
        round_kind<KIND>(v, f);
    }
}

// The first `count` of eight results to y[at]: codes, or fp32 that is rounded or not (`round`, uniform).  ROUNDED: the values are the format's.
template <int KIND, bool CODES, bool ROUNDED = false>
__device__ __forceinline__ void kind_store(void *y, int64_t at, int count, float (&v)[8], bool round, const ElemFormat &f)
{
    if constexpr (!ROUNDED) {
        if (CODES || round) round_kind<KIND>(v, f);
    }
    if constexpr (CODES) {
        const u32x4 w = encode_kind<KIND>(v, f);
        uint16_t *d = static_cast<uint16_t *>(y) + at;
        if (count >= 8) {
            *reinterpret_cast<u32x4_any2 *>(d) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) d[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
        }
    } else {
        float *d = static_cast<float *>(y) + at;
        if (count >= 8) {
            *reinterpret_cast<f32x4_any *>(d) = f32x4_any{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_any *>(d + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) d[i] = v[i];
        }
    }
}

// run(KIND, codes in, codes out) for a format and the tensors' types; formats without 16-bit codes have no codes.
template <class RUN>
void with_kind(const ElemFormat &f, int32_t store, int32_t result, RUN &&run)
{
    using std::integral_constant;
    const bool in = store == FMT_STORE_CODE16, out = result == FMT_RESULT_CODE16;
    auto types = [&](auto kind) {
        if (in && out) run(kind, std::true_type{}, std::true_type{});
        else if (in) run(kind, std::true_type{}, std::false_type{});
        else if (out) run(kind, std::false_type{}, std::true_type{});
        else run(kind, std::false_type{}, std::false_type{});
    };
    switch (elem_kind(f)) {
    case kKindNone: run(integral_constant<int, kKindNone>{}, std::false_type{}, std::false_type{}); break;
    case kKindMixed: run(integral_constant<int, kKindMixed>{}, std::false_type{}, std::false_type{}); break;
    case kKindHalf: types(integral_constant<int, kKindHalf>{}); break;
    case kKindMagic: types(integral_constant<int, kKindMagic>{}); break;
    default: types(integral_constant<int, kKindInteger>{}); break;
    }
}

}  // namespace fmt
