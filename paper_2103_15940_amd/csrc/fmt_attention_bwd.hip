// Attention, backward (fmt_attention.h has the mathematics and the layouts).
//
// P is made again from Q, K and lse.  Two kernels: one takes rows and adds up dQ over keys, the other takes keys and adds up dK and dV over
// rows, so that every sum is in one workgroup's accumulators, in a fixed order, at the price of S and dP twice (7 products instead of 5).
#include <type_traits>

#include "fmt_attention.h"

namespace fmt {

namespace {

struct AttnBwd {
    AttnShape s;
    AttnView q, k, v, o, go, dq, dk, dv;
    const float *lse;
    float *delta;             // [batch][heads][q_len]
    int32_t result;
    ElemFormat f;
};

// delta = sum over the head's columns of R(dO) O; eight lanes per row.
template <bool CODES>
__global__ __launch_bounds__(256) void attn_delta_kernel(AttnBwd a)
{
    const AttnShape &s = a.s;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 32 + (threadIdx.x >> 3), all = static_cast<int64_t>(s.batch) * s.heads * s.q_len;
    const int head = static_cast<int>(n % s.heads), t = static_cast<int>(n / s.heads % s.q_len), b = static_cast<int>(n / s.heads / s.q_len);
    float sum = 0.0f;
    if (n < all) {
        ElemFormat whole = a.f;
        whole.codec = CODES ? a.f.codec : kCodecNone;              // O is taken as it is
        for (int col = (threadIdx.x & 7) * 8; col < s.dim; col += 64) {
            const int count = min(s.dim - col, 8);
            float g[8], o[8];
            load8<CODES>(a.go.p, b * a.go.sb + t * a.go.st + head * a.go.sh + col, count, g, a.f);
            load8<CODES>(a.o.p, b * a.o.sb + t * a.o.st + head * a.o.sh + col, count, o, whole);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(g[j], o[j], sum);
        }
    }
#pragma unroll
    for (int w = 4; w > 0; w >>= 1) sum += __shfl_xor(sum, w);
    if (n < all && (threadIdx.x & 7) == 0) a.delta[(static_cast<int64_t>(b) * s.heads + head) * s.q_len + t] = sum;
}

// lse in base 2 with the sign that makes P of a row that sees nothing (lse = -inf) 0.
__device__ __forceinline__ float row_lse2(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

constexpr int kRowTile = 128, kKeyTile = 64;

template <int NQ, int NP, int DT, bool CODES, bool GCODES>
__global__ __launch_bounds__(256) void attn_dq_kernel(AttnBwd a)
{
    __shared__ AttnTile<NQ, DT, kKeyTile> ks, vs;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int b = blockIdx.z, kh = blockIdx.y;
    const AttnSeq seq = attn_seq(s, b);
    const int rows = s.q_len * s.group;
    const int row0 = blockIdx.x * kRowTile, row = row0 + wave * 32 + (lane & 31);
    const int t = row / s.group, head = kh * s.group + row % s.group;
    const bool live = row < rows;
    const int pos = seq.first + t;
    const int64_t i0 = static_cast<int64_t>(seq.first) + row0 / s.group;
    const int64_t i1 = static_cast<int64_t>(seq.first) + (min(row0 + kRowTile, rows) - 1) / s.group;

    u32x4 q[2 * DT][NQ], go[2 * DT][NQ];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half, count = live ? min(s.dim - col, 8) : 0;
        float v[8], g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = g[j] = 0.0f;
        if (count > 0) {
            load8<CODES>(a.q.p, b * a.q.sb + t * a.q.st + head * a.q.sh + col, count, v, a.f);
            load8<GCODES>(a.go.p, b * a.go.sb + t * a.go.st + head * a.go.sh + col, count, g, a.f);
        }
        bf16_pieces<NQ>(v, q[kk]);
        bf16_pieces<NQ>(g, go[kk]);
    }
    const int64_t at = (static_cast<int64_t>(b) * s.heads + head) * s.q_len + t;
    const float lse2 = live ? row_lse2(a.lse[at]) : INFINITY, delta = live ? a.delta[at] : 0.0f;

    f32x16 dq[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.0f;
    const int64_t kbase = b * a.k.sb + kh * a.k.sh, vbase = b * a.v.sb + kh * a.v.sh;
    const AttnTiles tiles = attn_tiles(s, seq.length, i0, i1, kKeyTile);
    for (int n = 0; n < tiles.count(); ++n) {
        const int k0 = tiles.at(n) * kKeyTile;
        __syncthreads();
        load_tokens<NQ, DT, kKeyTile, CODES>(ks, a.k.p, kbase, a.k.st, k0, seq.length, s.dim, a.f);
        load_tokens<NQ, DT, kKeyTile, CODES>(vs, a.v.p, vbase, a.v.st, k0, seq.length, s.dim, a.f);
        __syncthreads();
        const bool all = attn_sees_all(s, seq.length, i0, i1, k0, k0 + kKeyTile);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                u32x4 f[NQ];
                read_rows(ks, 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                x = mfma_pieces<NQ, NQ>(f, q[kk], x);
                read_rows(vs, 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                dp = mfma_pieces<NQ, NQ>(f, go[kk], dp);
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float ds[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = 8 * kb + j;
                    float y = x[i] * s.scale2;
                    if (!all && !attn_sees(s, seq.length, pos, k0 + 32 * kt + 8 * (i / 4) + 4 * half + (i & 3))) y = -INFINITY;
                    const float p = exp2_fast(y - lse2);
                    ds[j] = p == 0.0f ? 0.0f : p * (dp[i] - delta);
                }
                u32x4 pp[NP];
                bf16_pieces<NP>(ds, pp);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[NQ];
                    read_columns(ks, 32 * kt + 16 * kb, 32 * d, lane, f);
                    dq[d] = mfma_pieces<NQ, NP>(f, pp, dq[d]);
                }
            }
        }
    }
    if (!live) return;
    const int64_t base = b * a.dq.sb + t * a.dq.st + head * a.dq.sh;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = 32 * d + 8 * g + 4 * half;
            const float v[4] = {dq[d][4 * g] * s.scale, dq[d][4 * g + 1] * s.scale, dq[d][4 * g + 2] * s.scale, dq[d][4 * g + 3] * s.scale};
            store4(const_cast<void *>(a.dq.p), base + col, col, s.dim, v, a.result, a.f);
        }
}

constexpr int kKvKeys = 128, kKvRows = 32;

// Rows [row0, row0 + 32) of the heads that share a kv head, into a tile.
template <int NQ, int DT, bool CODES>
__device__ __forceinline__ void load_query_rows(AttnTile<NQ, DT, kKvRows> &t, const AttnView &x, const AttnShape &s, int b, int kh, int row0, int end,
                                                const ElemFormat &f)
{
    constexpr int kEights = 4 * DT, kAll = kKvRows * kEights;
#pragma unroll
    for (int i = 0; i < (kAll + 255) / 256; ++i) {
        const int n = threadIdx.x + 256 * i, r = n / kEights, col = (n % kEights) * 8, row = row0 + r;
        const int count = row < end ? min(s.dim - col, 8) : 0;
        float v[8];
        if (count > 0) {
            load8<CODES>(x.p, b * x.sb + (row / s.group) * x.st + (kh * s.group + row % s.group) * x.sh + col, count, v, f);
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

template <int NQ, int NP, int DT, bool CODES, bool GCODES>
__global__ __launch_bounds__(256) void attn_dkv_kernel(AttnBwd a)
{
    __shared__ AttnTile<NQ, DT, kKvRows> qs, gs;
    __shared__ float lses[kKvRows], deltas[kKvRows];
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int b = blockIdx.z, kh = blockIdx.y;
    const AttnSeq seq = attn_seq(s, b);
    const int k0 = blockIdx.x * kKvKeys, key = k0 + wave * 32 + (lane & 31);
    const bool live = key < s.k_len, used = key < seq.length;

    u32x4 k[2 * DT][NQ], v[2 * DT][NQ];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half, count = used ? min(s.dim - col, 8) : 0;
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = y[j] = 0.0f;
        if (count > 0) {
            load8<CODES>(a.k.p, b * a.k.sb + key * a.k.st + kh * a.k.sh + col, count, x, a.f);
            load8<CODES>(a.v.p, b * a.v.sb + key * a.v.st + kh * a.v.sh + col, count, y, a.f);
        }
        bf16_pieces<NQ>(x, k[kk]);
        bf16_pieces<NQ>(y, v[kk]);
    }
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;

    // tokens that may see one of these keys
    int64_t t0 = 0, t1 = s.q_len;
    if (s.causal) t0 = max(t0, static_cast<int64_t>(k0) - seq.first);
    if (s.window && k0 >= s.sinks) {
        t0 = max(t0, static_cast<int64_t>(k0) - s.window + 1 - seq.first);
        t1 = min(t1, static_cast<int64_t>(k0) + kKvKeys - 1 + s.window - seq.first);
    }
    if (k0 >= seq.length) t1 = 0;
    const int rows = s.q_len * s.group;
    const int first = t0 < t1 ? static_cast<int>(t0 * s.group / kKvRows * kKvRows) : 0, last = t0 < t1 ? static_cast<int>(t1 * s.group) : 0;
    for (int row0 = first; row0 < last; row0 += kKvRows) {
        __syncthreads();
        load_query_rows<NQ, DT, CODES>(qs, a.q, s, b, kh, row0, rows, a.f);
        load_query_rows<NQ, DT, GCODES>(gs, a.go, s, b, kh, row0, rows, a.f);
        if (threadIdx.x < kKvRows) {
            const int row = row0 + threadIdx.x;
            const bool there = row < rows;
            const int64_t at = (static_cast<int64_t>(b) * s.heads + kh * s.group + row % s.group) * s.q_len + row / s.group;
            lses[threadIdx.x] = there ? row_lse2(a.lse[at]) : INFINITY;
            deltas[threadIdx.x] = there ? a.delta[at] : 0.0f;
        }
        __syncthreads();
        f32x16 x, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 2 * DT; ++kk) {
            u32x4 f[NQ];
            read_rows(qs, lane & 31, 16 * kk + 8 * half, f);
            x = mfma_pieces<NQ, NQ>(f, k[kk], x);
            read_rows(gs, lane & 31, 16 * kk + 8 * half, f);
            dp = mfma_pieces<NQ, NQ>(f, v[kk], dp);
        }
        const int64_t i0 = static_cast<int64_t>(seq.first) + row0 / s.group;
        const int64_t i1 = static_cast<int64_t>(seq.first) + (min(row0 + kKvRows, rows) - 1) / s.group;
        const bool all = attn_sees_all(s, seq.length, i0, i1, k0, k0 + kKvKeys);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            float p[8], ds[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = 8 * kb + j, r = 8 * (i / 4) + 4 * half + (i & 3);
                float y = x[i] * s.scale2;
                if (!all && !attn_sees(s, seq.length, seq.first + (row0 + r) / s.group, key)) y = -INFINITY;
                p[j] = exp2_fast(y - lses[r]);
                ds[j] = p[j] == 0.0f ? 0.0f : p[j] * (dp[i] - deltas[r]);
            }
            u32x4 pp[NP], dd[NP];
            bf16_pieces<NP>(p, pp);
            bf16_pieces<NP>(ds, dd);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                u32x4 f[NQ];
                read_columns(gs, 16 * kb, 32 * d, lane, f);
                dv[d] = mfma_pieces<NQ, NP>(f, pp, dv[d]);
                read_columns(qs, 16 * kb, 32 * d, lane, f);
                dk[d] = mfma_pieces<NQ, NP>(f, dd, dk[d]);
            }
        }
    }
    if (!live) return;
    const int64_t kbase = b * a.dk.sb + key * a.dk.st + kh * a.dk.sh, vbase = b * a.dv.sb + key * a.dv.st + kh * a.dv.sh;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = 32 * d + 8 * g + 4 * half;
            const float x[4] = {dk[d][4 * g] * s.scale, dk[d][4 * g + 1] * s.scale, dk[d][4 * g + 2] * s.scale, dk[d][4 * g + 3] * s.scale};
            const float y[4] = {dv[d][4 * g], dv[d][4 * g + 1], dv[d][4 * g + 2], dv[d][4 * g + 3]};
            store4(const_cast<void *>(a.dk.p), kbase + col, col, s.dim, x, a.result, a.f);
            store4(const_cast<void *>(a.dv.p), vbase + col, col, s.dim, y, a.result, a.f);
        }
}

}  // namespace

int launch_attention_bwd(const AttnShape &s, const AttnView &q, const AttnView &k, const AttnView &v, const AttnView &o, const AttnView &go,
                         const float *lse, const AttnView &dq, const AttnView &dk, const AttnView &dv, int32_t store, int32_t result,
                         const ElemFormat &f, fmt_format_t fmt, hipStream_t stream)
{
    AttnBwd a{s, q, k, v, o, go, dq, dk, dv, lse, nullptr, result, f};
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len;
    int rc = get_acc_scratch(stream, static_cast<size_t>(all_rows) * sizeof(float), &a.delta);
    if (rc != FMT_OK) return rc;
    const bool gcodes = result == FMT_RESULT_CODE16;
    const dim3 delta_grid(static_cast<uint32_t>((all_rows + 31) / 32));
    if (all_rows == 0) a.s.q_len = 0;          // no queries: dK and dV are zero
    else if (gcodes) attn_delta_kernel<true><<<delta_grid, dim3(256), 0, stream>>>(a);
    else attn_delta_kernel<false><<<delta_grid, dim3(256), 0, stream>>>(a);
    const uint32_t row_tiles = static_cast<uint32_t>((static_cast<int64_t>(a.s.q_len) * s.group + kRowTile - 1) / kRowTile);
    const uint32_t key_tiles = static_cast<uint32_t>((s.k_len + kKvKeys - 1) / kKvKeys);
    const uint32_t kv_heads = static_cast<uint32_t>(s.kv_heads), batch = static_cast<uint32_t>(s.batch);
    with_attention(s.dim, store, result, fmt.m, [&](auto nq, auto np, auto dt, auto codes) {
        constexpr int NQ = decltype(nq)::value, NP = decltype(np)::value, DT = decltype(dt)::value;
        constexpr bool CODES = decltype(codes)::value;
        auto go2 = [&](auto g) {
            constexpr bool G = decltype(g)::value;
            if (row_tiles) attn_dq_kernel<NQ, NP, DT, CODES, G><<<dim3(row_tiles, kv_heads, batch), dim3(256), 0, stream>>>(a);
            if (key_tiles) attn_dkv_kernel<NQ, NP, DT, CODES, G><<<dim3(key_tiles, kv_heads, batch), dim3(256), 0, stream>>>(a);
        };
        if constexpr (NP != 3) {                 // three pieces: unrounded fp32 results, so fp32 gradients
            if (gcodes) {
                go2(std::true_type{});
                return;
            }
        }
        go2(std::false_type{});
    });
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
