// Row-wise operators of a transformer layer beside its products: dropout, and dropout + residual + layer norm, forward and backward.
//
//   forward    h = D(R(x)),  z = R(R(res) + h),  y = (z - mean) rstd R(gamma) + R(beta),
//              mean = sum z / N,  rstd = 1 / sqrt(sum (z - mean)^2 / N + eps)                        (N columns)
//   backward   xhat = (z - mean) rstd,  g = dy R(gamma),
//              dz = rstd (g - sum g / N - xhat sum(g xhat) / N),  dx = D(dz),
//              dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//   D          keeps an element where its 16 random bits are at least 65536 p, and multiplies it by 65536 / (65536 - 65536 p)
//
// The bits come from a counter (Philox-4x32 with ten rounds: J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", 2011), so the backward pass makes the same ones again and no mask is stored.  One call of the generator gives eight
// elements of a row their bits: 20 products of 32 x 32 bits, 2.5 per element, where 32 bits per element would take 5 and make the vector units
// the bound.
//
// A row is read once and stays in registers (8 columns per thread and piece): its mean and its squared deviations are two
// reductions over registers, in fp32.
#pragma once

#include "fmt_elem.h"

namespace fmt {

struct Drop {
    const uint64_t *rng;    // {seed, step}, or nullptr: nothing is dropped
    uint32_t site, least;   // an element is kept where its bits are >= least
    float scale;
};

struct DropKey {
    uint32_t k0, k1, step;
};

__device__ __forceinline__ DropKey drop_key(const Drop &d)
{
    const uint64_t seed = d.rng[0], step = d.rng[1];
    return DropKey{static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32), static_cast<uint32_t>(step)};
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// D of eight elements, the block-th eight of their tensor.
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t block, const DropKey &key, const Drop &d)
{
    uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32), c2 = key.step, c3 = d.site;
    uint32_t k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        const uint32_t n0 = xor3(static_cast<uint32_t>(b >> 32), c1, k0), n2 = xor3(static_cast<uint32_t>(a >> 32), c3, k1);
        c1 = static_cast<uint32_t>(b);
        c3 = static_cast<uint32_t>(a);
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = (i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
        // rounded on its own (no fused multiply-add with what follows): the same in forward, backward and any other order
        v[i] = bits >= d.least ? __fmul_rn(v[i], d.scale) : 0.0f;
    }
}

inline Drop make_drop(const fmt_dropout_t &d)
{
    const uint32_t least = static_cast<uint32_t>(static_cast<double>(d.p) * 65536.0 + 0.5);
    const float scale = least < 65536u ? static_cast<float>(65536.0 / (65536.0 - least)) : 0.0f;
    return Drop{d.p > 0.0f ? d.rng : nullptr, d.site, least, scale};
}

// Sum over the T threads of a row: T <= 64 are neighbouring lanes of a wave, more are T / 64 waves of a workgroup with several such rows.
template <int T>
__device__ __forceinline__ float row_sum(float s, float *shared)
{
#pragma unroll
    for (int w = (T < 64 ? T : 64) / 2; w > 0; w >>= 1) s += __shfl_xor(s, w);
    if constexpr (T > 64) {
        __syncthreads();                                  // what the sum before left there has been read
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
        __syncthreads();
        const int first = threadIdx.x / T * (T / 64);
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) s += shared[first + w];
    }
    return s;
}

// Parameters of eight columns, rounded.
template <int KIND>
__device__ __forceinline__ void load_weight(const float *w, int col, int count, float other, float (&v)[8], const ElemFormat &f)
{
    if (w) {
        kind_values<KIND, false>(raw_load<false>(w, col, count), v, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = other;
    }
}

// run(threads per row, eights per thread) for rows of so many columns: the fewest threads that hold the row with at most two eights each,
// so that several rows fill a workgroup; beyond 4096 columns a whole workgroup of 1024 and up to four.
template <class RUN>
void with_shape(int64_t cols, RUN &&run)
{
    using std::integral_constant;
    if (cols <= 128) run(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (cols <= 512) run(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (cols <= 1024) run(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (cols <= 2048) run(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (cols <= 4096) run(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (cols <= 8192) run(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    else if (cols <= 16384) run(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else run(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

}  // namespace fmt
