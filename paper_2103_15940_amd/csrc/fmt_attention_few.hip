// Attention of few rows (a query head or two, single tokens) over many keys: read keys and values once, as fast as they come.
//
// With at most 8 rows per (batch, kv head) the matrix cores have nothing to do (a 32 x 32 tile would be three quarters padding), and what bounds the
// call is the bytes of K and V: 2 bytes per element in codes, for which the vector units have about 100 instructions per 8 elements of both.
// So: 4 DT lanes hold a key's 32 DT columns, 8 each; a wave has 64 / (4 DT) keys at a time, and U such groups of K and V in flight. A lane
// forms its 8 columns' part of the scores, the lanes of a key add them up with DPP (no LDS), and every group of lanes keeps its own
// running maximum, sum and outputs, which meet in LDS at the end. The keys of a sequence are cut in parts for enough workgroups; a second
// kernel joins them. All of it is fp32: any operand of any format is exact.
//
// Measured: one head per kv head (8 of 128, 32768 keys in bfloat16, 134 MB) 23 us, 5.8 TB/s; four (48 sequences of up to 8191 keys, 4 kv heads
// of 64, 1/6/9 codes, 197 MB) 52 us, 3.8 TB/s, bound by vector issue: 16 fused multiply-adds, 3 DPP additions and an exponential per
// row and 8 elements of K and V, beside 16 instructions of decoding.
//
// Codes become fp32 by their bits: sign, and exponent field and mantissa at the place of fp32's, times 2^(127 - bias); the code's denormals are
// fp32 denormals then, and right too. For 1/6/9 the factors are left to Q (2^64), the scale (2^32) and the outputs (2^96), and P meets V
// times 2^64, so that sums stay among the normal numbers: multiplied after the exponential, since a 64 added in its argument would
// take five bits from it.
#include <algorithm>
#include <type_traits>

#include "fmt_attention.h"

namespace fmt {

namespace {

struct AttnFew {
    AttnShape s;
    AttnView q, k, v, o;
    float *lse;               // [batch][heads][q_len]
    int32_t result, splits;
    bool codes;
    float *part;              // splits > 1: [splits][batch * heads * q_len][dim] normalised outputs, then as many maxima in base 2, then sums
    float factor;             // 2^(127 - bias)
    uint32_t body;            // magnitude bits of a code, in both halves of a word
    ElemFormat f;
};

enum : int { kFewFloat = 0, kFewCodes = 1, kFewSix = 2, kFewBf16 = 3, kFewHalf = 4 };

template <int CONTROL>
__device__ __forceinline__ float dpp_add(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xF, 0xF, true));
}

// Sum over 8 (or 16) neighbouring lanes, in all of them: pairs, quads, halves of a row of 16, the row.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x)
{
    x = dpp_add<0xB1>(x);
    x = dpp_add<0x4E>(x);
    x = dpp_add<0x141>(x);
    if constexpr (LANES == 16) x = dpp_add<0x140>(x);
    return x;
}

template <int KIND>
__device__ __forceinline__ void few_values(const RawEight<KIND != kFewFloat> &r, float (&v)[8], const AttnFew &a, uint32_t &high)
{
    if constexpr (KIND == kFewFloat) {
        raw_values<false>(r, v, a.f);
    } else if constexpr (KIND == kFewBf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r.w[0][i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[0][i] & 0xFFFF0000u);
        }
    } else if constexpr (KIND == kFewHalf) {
        const f16x8 h = __builtin_bit_cast(f16x8, r.w[0]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(h[i]);
    } else {
        u16x2 top = __builtin_bit_cast(u16x2, high);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = r.w[0][i];
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w & a.body));
            if constexpr (KIND == kFewSix) {              // 1/6/9: sign extended, exponent and mantissa from bit 14 on
                v[2 * i] = __int_as_float((static_cast<int>(w << 16) >> 2) & 0x9FFFFFFF);
                v[2 * i + 1] = __int_as_float((static_cast<int>(w) >> 2) & 0x9FFFC000);
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t c = w >> (16 * j);
                    v[2 * i + j] = __uint_as_float((c & a.body & 0xFFFFu) << a.f.p.shift | (c >> a.f.p.sign_pos & 1u) << 31) * a.factor;
                }
            }
        }
        high = __builtin_bit_cast(uint32_t, top);
    }
}

// Groups of keys in flight per wave: as many as leave four workgroups their registers in a compute unit (three with 2 or 4 rows, two with 8).
template <int R, int KIND>
constexpr int kFewGroups = KIND == kFewFloat || R > 2 ? 2 : 4;

template <int R, int DT, int KIND>
__global__ __launch_bounds__(256, R <= 1 ? 4 : R <= 4 ? 3 : 2) void attn_few_kernel(AttnFew a)
{
    constexpr int LANES = 4 * DT, SLOTS = 64 / LANES, U = kFewGroups<R, KIND>, TILE = 4 * U * SLOTS, DP = 32 * DT;
    constexpr bool CODES = KIND != kFewFloat;
    __shared__ alignas(16) float outs[4 * SLOTS][R][DP];
    __shared__ float tops[4 * SLOTS][R], sums[4 * SLOTS][R];
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = lane / LANES, col = (lane % LANES) * 8, have = s.dim - col;
    const uint32_t id = xcd_order(blockIdx.x, gridDim.x);
    const int split = static_cast<int>(id % a.splits), kh = static_cast<int>(id / a.splits % s.kv_heads), b = static_cast<int>(id / a.splits / s.kv_heads);
    const AttnSeq seq = attn_seq(s, b);
    const int rows = s.q_len * s.group;
    const int64_t i0 = seq.first, i1 = static_cast<int64_t>(seq.first) + s.q_len - 1;
    const AttnTiles tiles = attn_tiles(s, seq.length, i0, i1, TILE);
    const int count = tiles.count();
    const int begin = static_cast<int>(static_cast<int64_t>(count) * split / a.splits);
    const int end = static_cast<int>(static_cast<int64_t>(count) * (split + 1) / a.splits);
    const int64_t kbase = b * a.k.sb + kh * a.k.sh + col, vbase = b * a.v.sb + kh * a.v.sh + col;

    RawEight<CODES> kr[U], vr[U];
    const int mine = wave * U * SLOTS + slot;             // the lane's keys of a tile: mine, mine + SLOTS, ...
    auto fetch = [&](int n) __attribute__((always_inline)) {
        const int k0 = tiles.at(n) * TILE + mine;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = k0 + u * SLOTS, there = key < seq.length ? have : 0;
            kr[u] = raw_load<CODES>(a.k.p, kbase + key * a.k.st, there);
            vr[u] = raw_load<CODES>(a.v.p, vbase + key * a.v.st, there);
        }
    };
    if (begin < end) fetch(begin);
    float q[R][8], o[R][8], top[R], sum[R];
    AttnKeys sees[R];
    // Q takes the scale's sign, so that products are ordered as the scores are; a scale of 0 makes Q zero
    const float scale2 = s.scale2 == 0.0f ? 1.0f : fabsf(s.scale2) * (KIND == kFewSix ? 0x1p32f : 1.0f);
    const float sign = (KIND == kFewSix ? 0x1p64f : 1.0f) * (s.scale2 > 0.0f ? 1.0f : s.scale2 < 0.0f ? -1.0f : 0.0f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = r / s.group, head = kh * s.group + r % s.group;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[r][j] = o[r][j] = 0.0f;
        if (r < rows && have > 0) load8_any(a.q.p, b * a.q.sb + t * a.q.st + head * a.q.sh + col, min(have, 8), q[r], a.codes, a.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[r][j] *= sign;
        top[r] = -INFINITY;
        sum[r] = 0.0f;
        sees[r] = attn_keys(s, seq.length, seq.first + t);
    }
    uint32_t high = 0;
    for (int n = begin; n < end; ++n) {
        const int tile0 = tiles.at(n) * TILE, k0 = tile0 + mine;
        float x[U][R], v[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float k[8];
            few_values<KIND>(kr[u], k, a, high);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float d = k[0] * q[r][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) d = fmaf(k[j], q[r][j], d);
                x[u][r] = lanes_sum<LANES>(d);
            }
            few_values<KIND>(vr[u], v[u], a, high);
        }
        if (n + 1 < end) fetch(n + 1);
        if (!attn_sees_all(s, seq.length, i0, i1, tile0, tile0 + TILE)) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int key = k0 + u * SLOTS;
                    const bool seen = static_cast<uint32_t>(key - sees[r].first) < sees[r].count || key < sees[r].sinks;
                    x[u][r] = seen ? x[u][r] : -INFINITY;
                }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float next = top[r];
#pragma unroll
            for (int u = 0; u < U; ++u) next = fmaxf(next, x[u][r]);
            // the maximum's product is rounded once, for all uses: an unrounded one in one of them, times all tiles, is a drift
            float before = top[r] * scale2, base = next == -INFINITY ? 0.0f : next * scale2;
            asm("" : "+v"(before), "+v"(base));
            const float shrink = exp2_fast(before - base);
            top[r] = next;
            sum[r] *= shrink;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[r][j] *= shrink;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float p = exp2_fast(fmaf(x[u][r], scale2, -base));
                sum[r] += p;
                if constexpr (KIND == kFewSix) p *= 0x1p64f;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[r][j] = fmaf(p, v[u][j], o[r][j]);
            }
        }
    }
    // codes of infinities and NaN, which their bits do not show as such, make NaN
    bool bad = false;
    if constexpr (KIND == kFewCodes || KIND == kFewSix) bad = max(high >> 16, high & 0xFFFFu) >= a.f.p.top_code;
    const int at = wave * SLOTS + slot;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int j = 0; j < 8; j += 4) *reinterpret_cast<f32x4 *>(&outs[at][r][col + j]) = f32x4{o[r][j], o[r][j + 1], o[r][j + 2], o[r][j + 3]};
        if (lane % LANES == 0) {
            tops[at][r] = top[r] * scale2;
            sums[at][r] = sum[r];
        }
    }
    bad = __syncthreads_or(bad);
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len;
    for (int n = threadIdx.x; n < R * DP; n += 256) {
        const int r = n / DP, c = n % DP;
        if (r >= rows || c >= s.dim) continue;
        float high_top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4 * SLOTS; ++i) high_top = fmaxf(high_top, tops[i][r]);
        const float base = high_top == -INFINITY ? 0.0f : high_top;
        float total = 0.0f, out = 0.0f;
#pragma unroll
        for (int i = 0; i < 4 * SLOTS; ++i) {
            const float w = exp2_fast(tops[i][r] - base);
            total = fmaf(w, sums[i][r], total);
            out = fmaf(w, outs[i][r][c], out);
        }
        if (bad) total = out = NAN;
        out = total == 0.0f ? 0.0f : out / total;
        if constexpr (KIND == kFewSix) out *= 0x1p32f;
        const int t = r / s.group, head = kh * s.group + r % s.group;
        const int64_t row = (static_cast<int64_t>(b) * s.heads + head) * s.q_len + t;
        if (a.splits > 1) {
            a.part[(split * all_rows + row) * s.dim + c] = out;
            if (c == 0) {
                float *records = a.part + a.splits * all_rows * s.dim + split * all_rows + row;
                records[0] = high_top;
                records[a.splits * all_rows] = total;
            }
        } else {
            const float y[4] = {out, 0.0f, 0.0f, 0.0f};
            store4(const_cast<void *>(a.o.p), b * a.o.sb + t * a.o.st + head * a.o.sh + c, 1, y, a.result, a.f);
            if (c == 0 && a.lse) a.lse[row] = lse_of(high_top, total);
        }
    }
}

template <int R, int DT>
void launch_few(const AttnFew &a, fmt_format_t f, dim3 grid, hipStream_t stream)
{
    const dim3 threads(256);
    if (!a.codes) attn_few_kernel<R, DT, kFewFloat><<<grid, threads, 0, stream>>>(a);
    else if (a.f.codec == kCodecBf16) attn_few_kernel<R, DT, kFewBf16><<<grid, threads, 0, stream>>>(a);
    else if (f.e == 5 && f.m == 10) attn_few_kernel<R, DT, kFewHalf><<<grid, threads, 0, stream>>>(a);
    else if (f.e == 6 && f.m == 9) attn_few_kernel<R, DT, kFewSix><<<grid, threads, 0, stream>>>(a);
    else attn_few_kernel<R, DT, kFewCodes><<<grid, threads, 0, stream>>>(a);
}

}  // namespace

int attention_few_tile(int rows, int dim, int32_t store) { return 4 * (store == FMT_STORE_CODE16 && rows <= 2 ? 4 : 2) * (dim <= 64 ? 8 : 4); }

int launch_attention_few(const AttnShape &s, const AttnView &q, const AttnView &k, const AttnView &v, const AttnView &o, float *lse, int32_t store,
                         int32_t result, int32_t splits, float *part, const ElemFormat &f, fmt_format_t fmt, hipStream_t stream)
{
    const uint32_t body = (1u << (fmt.e + fmt.m)) - 1u;
    const int bias = (1 << (fmt.e - 1)) - 1;
    const AttnFew a{s, q, k, v, o, lse, result, splits, store == FMT_STORE_CODE16, part, ldexpf(1.0f, 127 - bias), body * 0x10001u, f};
    const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(s.batch) * s.kv_heads * splits));
    const int rows = s.q_len * s.group;
    auto go = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (rows <= 1) launch_few<1, DT>(a, fmt, grid, stream);
        else if (rows <= 2) launch_few<2, DT>(a, fmt, grid, stream);
        else if (rows <= 4) launch_few<4, DT>(a, fmt, grid, stream);
        else launch_few<8, DT>(a, fmt, grid, stream);
    };
    with_dim(s.dim, go);
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
