// Runs of consecutive elements of the row-wise and attention kernels: fp32 values that are rounded to the format as they are read, or
// the format's own 16-bit codes; and results as unrounded fp32, rounded fp32 or codes.
#pragma once

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
        for (int i = 0; i < N; ++i) v[i] = static_cast<float>(static_cast<_Float16>(v[i]));
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

// The first `count` of eight results to y[at].  RESULT: FMT_RESULT_*; ROUNDED: the values are the format's already.
template <int RESULT, bool ROUNDED = false>
__device__ __forceinline__ void store8(void *y, int64_t at, int count, float (&v)[8], const ElemFormat &f)
{
    if (RESULT != FMT_RESULT_F32 && !ROUNDED) round_values(v, f);
    if constexpr (RESULT == FMT_RESULT_CODE16) {
        uint16_t c[8];
        encode_values(v, c, f);
        uint16_t *d = static_cast<uint16_t *>(y) + at;
        if (count >= 8) {
            u16x8_any w;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = c[i];
            *reinterpret_cast<u16x8_any *>(d) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) d[i] = c[i];
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

// The same with the type known at run time (uniform).
__device__ __forceinline__ void load8_any(const void *x, int64_t at, int count, float (&v)[8], bool codes, const ElemFormat &f)
{
    if (codes) load8<true>(x, at, count, v, f);
    else load8<false>(x, at, count, v, f);
}

}  // namespace fmt
