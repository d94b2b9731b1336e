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
#include <type_traits>

#include "fmt_elem.h"

namespace fmt {

namespace {

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

// D of eight elements, the block-th eight of their tensor.
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t block, const DropKey &key, const Drop &d)
{
    uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32), c2 = key.step, c3 = d.site;
    uint32_t k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        const uint32_t n0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0, n2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
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

// ------------------------------------------------------------------ dropout

constexpr int kDropThreads = 256, kDropRuns = 4;      // eights per thread

template <bool CODES, int RESULT>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const void *x, int64_t ldx, void *y, int64_t ldy, int64_t rows,
                                                                int64_t cols, uint32_t blocks, Drop d, ElemFormat f)
{
    const uint64_t total = static_cast<uint64_t>(rows) * blocks, first = static_cast<uint64_t>(blockIdx.x) * (kDropThreads * kDropRuns);
    const uint64_t row0 = first / blocks;
    const uint32_t at0 = static_cast<uint32_t>(first - row0 * blocks);
    const DropKey key = drop_key(d);
#pragma unroll
    for (int i = 0; i < kDropRuns; ++i) {
        const uint32_t step = threadIdx.x + kDropThreads * i;
        const uint64_t n = first + step;
        if (n >= total) break;
        const uint32_t past = at0 + step, over = past / blocks, g = past - over * blocks;
        const int64_t row = static_cast<int64_t>(row0 + over), col = static_cast<int64_t>(g) * 8;
        const int count = static_cast<int>(cols - col < 8 ? cols - col : 8);
        float v[8];
        load8<CODES>(x, row * ldx + col, count, v, f);
        drop8(v, n, key, d);
        store8<RESULT>(y, row * ldy + col, count, v, f);
    }
}

// ------------------------------------------------------------------ sums over the threads of a row

// T threads of one row: T <= 64 are neighbouring lanes of a wave, more are the whole workgroup.
template <int T>
__device__ __forceinline__ float row_sum(float s, float *shared)
{
#pragma unroll
    for (int w = (T < 64 ? T : 64) / 2; w > 0; w >>= 1) s += __shfl_xor(s, w);
    if constexpr (T > 64) {
        __syncthreads();                                  // what the sum before left there has been read
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) s += shared[w];
    }
    return s;
}

struct NormFwd {
    const void *x, *res;
    const float *gamma, *beta;
    void *z, *y;
    float *mean, *rstd;
    int64_t rows, ldx, ldres, ldz, ldy;
    int32_t cols;
    float eps;
    Drop drop;
    ElemFormat f;
};

// Parameters of eight columns, rounded.
__device__ __forceinline__ void load_weight(const float *w, int col, int count, float other, float (&v)[8], const ElemFormat &f)
{
    if (w) {
        load8<false>(w, col, count, v, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = other;
    }
}

template <int T, int V>
constexpr int kNormThreads = T < 256 ? 256 : T;

template <int T, int V, bool CODES, int RESULT>
__global__ __launch_bounds__((kNormThreads<T, V>)) void norm_fwd_kernel(NormFwd a)
{
    __shared__ float shared[T > 64 ? T / 64 : 1];
    constexpr int kRows = kNormThreads<T, V> / T;
    const int t = threadIdx.x % T;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / T;
    const bool live = row < a.rows;                       // no early exit: lanes of one wave add up together
    const int blocks = (a.cols + 7) >> 3;
    float z[V][8];
    float sum = 0.0f;
    DropKey key{};
    if (a.drop.rng) key = drop_key(a.drop);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = t + T * i, col = g * 8;
        const int count = live ? min(a.cols - col, 8) : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] = 0.0f;
        if (count > 0) {
            load8<CODES>(a.x, row * a.ldx + col, count, z[i], a.f);
            if (a.drop.rng) drop8(z[i], static_cast<uint64_t>(row) * blocks + g, key, a.drop);
            if (a.res) {
                float r[8];
                load8<CODES>(a.res, row * a.ldres + col, count, r, a.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) z[i][j] = __fadd_rn(r[j], z[i][j]);
            }
            if (a.res || a.drop.rng) round_values(z[i], a.f);       // (what lies past the last column is 0 and stays it)
            if (a.z) store8<RESULT, true>(a.z, row * a.ldz + col, count, z[i], a.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += z[i][j];
        }
    }
    const float mean = row_sum<T>(sum, shared) / static_cast<float>(a.cols);
    float square = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int count = live ? min(a.cols - (t + T * i) * 8, 8) : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float c = z[i][j] - mean;
            square += j < count ? c * c : 0.0f;
        }
    }
    const float var = row_sum<T>(square, shared) / static_cast<float>(a.cols);
    const float rstd = 1.0f / sqrtf(var + a.eps);
    if (live && t == 0 && a.mean) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int col = (t + T * i) * 8;
        const int count = live ? min(a.cols - col, 8) : 0;
        if (count > 0) {
            float w[8], b[8], y[8];
            load_weight(a.gamma, col, count, 1.0f, w, a.f);
            load_weight(a.beta, col, count, 0.0f, b, a.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = fmaf((z[i][j] - mean) * rstd, w[j], b[j]);
            store8<RESULT>(a.y, row * a.ldy + col, count, y, a.f);
        }
    }
}

struct NormBwd {
    const void *dy, *z;
    const float *mean, *rstd, *gamma;
    void *dz, *dx;
    float *partial;          // [workgroups][2][cols], or nullptr: no parameter gradients
    int64_t rows, lddy, ldz, lddz, lddx;
    int32_t cols;
    Drop drop;
    ElemFormat f;
};

// A workgroup takes rows blockIdx, blockIdx + gridDim, ... (by kRows) and keeps the parameters' gradients of its columns in registers; at
// the end its threads add them up and write one record, and norm_param_kernel adds the records in a fixed order.
template <int T, int V, bool CODES, int RESULT>
__global__ __launch_bounds__((kNormThreads<T, V>)) void norm_bwd_kernel(NormBwd a)
{
    constexpr int kThreads = kNormThreads<T, V>, kRows = kThreads / T;
    __shared__ float shared[T > 64 ? T / 64 : 1];
    __shared__ float joined[kRows > 1 ? kThreads * 8 : 1];
    const int t = threadIdx.x % T, mine = threadIdx.x / T;
    const int blocks = (a.cols + 7) >> 3;
    const float n = 1.0f / static_cast<float>(a.cols);
    float w[V][8], dw[V][8], db[V][8];
    DropKey key{};
    if (a.drop.rng) key = drop_key(a.drop);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int col = (t + T * i) * 8, count = min(a.cols - col, 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[i][j] = dw[i][j] = db[i][j] = 0.0f;
        if (count > 0) load_weight(a.gamma, col, count, 1.0f, w[i], a.f);
    }
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.rows; base += static_cast<int64_t>(gridDim.x) * kRows) {
        const int64_t row = base + mine;
        const bool live = row < a.rows;
        const float mean = live ? a.mean[row] : 0.0f, rstd = live ? a.rstd[row] : 0.0f;
        float g[V][8], xhat[V][8];
        float sum = 0.0f, along = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int col = (t + T * i) * 8, count = live ? min(a.cols - col, 8) : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[i][j] = xhat[i][j] = 0.0f;
            if (count > 0) {
                load8<CODES>(a.dy, row * a.lddy + col, count, g[i], a.f);
                load8<CODES>(a.z, row * a.ldz + col, count, xhat[i], a.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    xhat[i][j] = j < count ? (xhat[i][j] - mean) * rstd : 0.0f;
                    dw[i][j] = fmaf(g[i][j], xhat[i][j], dw[i][j]);
                    db[i][j] += g[i][j];
                    g[i][j] *= w[i][j];
                    sum += g[i][j];
                    along = fmaf(g[i][j], xhat[i][j], along);
                }
            }
        }
        const float m0 = row_sum<T>(sum, shared) * n, m1 = row_sum<T>(along, shared) * n;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int gi = t + T * i, col = gi * 8, count = live ? min(a.cols - col, 8) : 0;
            if (count > 0) {
                float d[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = rstd * (g[i][j] - m0 - xhat[i][j] * m1);
                if (a.dx) {
                    float e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] = d[j];
                    if (a.drop.rng) drop8(e, static_cast<uint64_t>(row) * blocks + gi, key, a.drop);
                    store8<RESULT>(a.dx, row * a.lddx + col, count, e, a.f);
                }
                store8<RESULT>(a.dz, row * a.lddz + col, count, d, a.f);
            }
        }
    }
    if (!a.partial) return;
    float *record = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = which ? db[i][j] : dw[i][j];
            if constexpr (kRows > 1) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) joined[j * kThreads + threadIdx.x] = s[j];
                __syncthreads();
                if (mine == 0) {
#pragma unroll
                    for (int r = 1; r < kRows; ++r)
#pragma unroll
                        for (int j = 0; j < 8; ++j) s[j] += joined[j * kThreads + r * T + t];
                }
            }
            const int col = (t + T * i) * 8;
            if (mine == 0)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < a.cols) record[which * a.cols + col + j] = s[j];
        }
    }
}

// dgamma and dbeta from the workgroups' records: 64 columns per workgroup, 16 threads share a column's records.
__global__ __launch_bounds__(1024) void norm_param_kernel(const float *partial, int records, int cols, float *dgamma, float *dbeta)
{
    __shared__ float part[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), lane = threadIdx.x >> 6, width = 2 * cols;
    float s = 0.0f;
    if (c < width)
        for (int r = lane; r < records; r += 16) s += partial[static_cast<int64_t>(r) * width + c];
    part[lane][threadIdx.x & 63] = s;
    __syncthreads();
    if (lane == 0 && c < width) {
#pragma unroll
        for (int r = 1; r < 16; ++r) s += part[r][threadIdx.x & 63];
        if (c < cols) dgamma[c] = s;
        else dbeta[c - cols] = s;
    }
}

Drop make_drop(const fmt_dropout_t &d)
{
    const uint32_t least = static_cast<uint32_t>(static_cast<double>(d.p) * 65536.0 + 0.5);
    const float scale = least < 65536u ? static_cast<float>(65536.0 / (65536.0 - least)) : 0.0f;
    return Drop{d.p > 0.0f ? d.rng : nullptr, d.site, least, scale};
}

// run(codes, result) with both as compile-time values.
template <class RUN>
void with_types(int32_t store, int32_t result, RUN &&run)
{
    auto r = [&](auto codes) {
        if (result == FMT_RESULT_F32) run(codes, std::integral_constant<int, FMT_RESULT_F32>{});
        else if (result == FMT_RESULT_ROUND) run(codes, std::integral_constant<int, FMT_RESULT_ROUND>{});
        else run(codes, std::integral_constant<int, FMT_RESULT_CODE16>{});
    };
    if (store == FMT_STORE_CODE16) r(std::true_type{});
    else r(std::false_type{});
}

// run(threads per row, eights per thread) for rows of so many columns: the fewest threads that hold the row with at most two eights each,
// so that several rows fill a workgroup of 256; beyond 4096 columns a whole workgroup of 1024 and up to eight.
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

}  // namespace

int launch_dropout(const void *x, int64_t ldx, void *y, int64_t ldy, int64_t rows, int64_t cols, const fmt_dropout_t &d, int32_t store,
                   int32_t result, const ElemFormat &f, hipStream_t stream)
{
    Drop drop = make_drop(d);
    drop.rng = d.rng;
    const uint32_t blocks = static_cast<uint32_t>((cols + 7) / 8);
    const uint64_t grid = (static_cast<uint64_t>(rows) * blocks + kDropThreads * kDropRuns - 1) / (kDropThreads * kDropRuns);
    if (grid > 0x7FFFFFFFull) return FMT_ERR_SHAPE;
    with_types(store, result, [&](auto codes, auto res) {
        dropout_kernel<decltype(codes)::value, decltype(res)::value>
            <<<dim3(static_cast<uint32_t>(grid)), dim3(kDropThreads), 0, stream>>>(x, ldx, y, ldy, rows, cols, blocks, drop, f);
    });
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

int launch_layernorm_fwd(const LayerNorm &n, const void *x, int64_t ldx, const void *res, int64_t ldres, const float *gamma,
                         const float *beta, float eps, void *z, int64_t ldz, void *y, int64_t ldy, float *mean, float *rstd,
                         const ElemFormat &f, hipStream_t stream)
{
    const NormFwd a{x, res, gamma, beta, z, y, mean, rstd, n.rows, ldx, ldres, ldz, ldy, static_cast<int32_t>(n.cols), eps,
                    make_drop(n.drop), f};
    int rc = FMT_OK;
    with_shape(n.cols, [&](auto threads, auto eights) {
        constexpr int T = decltype(threads)::value, V = decltype(eights)::value, kThreads = kNormThreads<T, V>;
        const int64_t grid = (n.rows + kThreads / T - 1) / (kThreads / T);
        if (grid > 0x7FFFFFFF) {
            rc = FMT_ERR_SHAPE;
            return;
        }
        with_types(n.store, n.result, [&](auto codes, auto result) {
            norm_fwd_kernel<T, V, decltype(codes)::value, decltype(result)::value>
                <<<dim3(static_cast<uint32_t>(grid)), dim3(kThreads), 0, stream>>>(a);
        });
    });
    if (rc != FMT_OK) return rc;
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

int launch_layernorm_bwd(const LayerNorm &n, const void *dy, int64_t lddy, const void *z, int64_t ldz, const float *mean,
                         const float *rstd, const float *gamma, void *dz, int64_t lddz, void *dx, int64_t lddx, float *dgamma,
                         float *dbeta, const ElemFormat &f, hipStream_t stream)
{
    int cus = 0;
    int rc = device_cu_count(&cus);
    if (rc != FMT_OK) return rc;
    NormBwd a{dy, z, mean, rstd, gamma, dz, dx, nullptr, n.rows, lddy, ldz, lddz, lddx, static_cast<int32_t>(n.cols),
              make_drop(n.drop), f};
    int records = 0;
    with_shape(n.cols, [&](auto threads, auto eights) {
        constexpr int T = decltype(threads)::value, V = decltype(eights)::value, kThreads = kNormThreads<T, V>;
        const int64_t want = (n.rows + kThreads / T - 1) / (kThreads / T);
        const int most = cus * (1024 / kThreads);
        records = static_cast<int>(want < most ? want : most);
        if (records == 0) return;
        if (dgamma) {
            rc = get_acc_scratch(stream, static_cast<size_t>(records) * 2 * static_cast<size_t>(n.cols) * sizeof(float), &a.partial);
            if (rc != FMT_OK) return;
        }
        with_types(n.store, n.result, [&](auto codes, auto result) {
            norm_bwd_kernel<T, V, decltype(codes)::value, decltype(result)::value>
                <<<dim3(static_cast<uint32_t>(records)), dim3(kThreads), 0, stream>>>(a);
        });
    });
    if (rc != FMT_OK) return rc;
    if (dgamma)
        norm_param_kernel<<<dim3(static_cast<uint32_t>((2 * n.cols + 63) / 64)), dim3(1024), 0, stream>>>(
            a.partial, records, static_cast<int>(n.cols), dgamma, dbeta);
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
