// Dropout, residual and layer norm, backward (fmt_norm.h has the mathematics).
//
// A workgroup takes rows blockIdx, blockIdx + gridDim, ... (by kRows) and keeps the parameters' gradients of its columns in registers,
// while the next row's elements are on their way; at the end its rows add theirs up in LDS and write one record, and norm_param_kernel
// adds the records in a fixed order.  (Atomic additions would save that kernel, and give other bits every time.)
//
// Measured: 50001 x 768 in fp32, 461 MB: 91 us, 5.1 TB/s, and 4 to 5 us for the records; bound by memory.  4096 x 1024 in bfloat16: 15 us and 4,
// two rows per wave, one after the other, with eight waves on a compute unit.
#include "fmt_norm.h"

namespace fmt {

namespace {

struct NormBwd {
    const void *dy, *z;
    const float *mean, *rstd, *gamma;
    void *dz, *dx;
    float *partial;          // [workgroups][2][cols], or nullptr: no parameter gradients
    int64_t rows, lddy, ldz, lddz, lddx;
    int32_t cols;
    bool round;              // whether fp32 results are rounded
    Drop drop;
    ElemFormat f;
};

template <int T>
constexpr int kNormThreads = T < 512 ? 512 : T;

template <int T, int V, int KIND, bool CODES, bool OUT>
__global__ __launch_bounds__(kNormThreads<T>, T == 1024 ? 4 : 2) void norm_bwd_kernel(NormBwd a)
{
    constexpr int kThreads = kNormThreads<T>, kRows = kThreads / T, kWidth = 8 * T;
    constexpr bool kAhead = V <= 2 && T < 1024;           // registers for the next row's elements
    __shared__ float shared[T > 64 ? kThreads / 64 : 1];
    __shared__ float joined[kRows > 1 ? kRows : 1][kRows > 1 ? kWidth : 1];
    const int t = threadIdx.x % T, mine = threadIdx.x / T;
    const int blocks = (a.cols + 7) >> 3;
    const float n = 1.0f / static_cast<float>(a.cols);
    RawEight<CODES> dr[V], zr[V];
    float mean = 0.0f, rstd = 0.0f;
    auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        const bool live = row < a.rows;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int col = (t + T * i) * 8, count = live ? a.cols - col : 0;
            dr[i] = raw_load<CODES>(a.dy, row * a.lddy + col, count);
            zr[i] = raw_load<CODES>(a.z, row * a.ldz + col, count);
        }
        mean = live ? a.mean[row] : 0.0f;
        rstd = live ? a.rstd[row] : 0.0f;
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
    int64_t base = static_cast<int64_t>(blockIdx.x) * kRows;
    fetch(base + mine);
    constexpr bool kHold = T < 1024;                      // registers for the weights
    float w[kHold ? V : 1][8], dw[V][8], db[V][8];
    DropKey key{};
    if (a.drop.rng) key = drop_key(a.drop);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (kHold) load_weight<KIND>(a.gamma, (t + T * i) * 8, a.cols - (t + T * i) * 8, 1.0f, w[i], a.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.0f;
    }
    for (; base < a.rows; base += step) {
        const int64_t row = base + mine;
        const bool live = row < a.rows;
        const float scale = rstd, centre = mean;
        float g[V][8], xhat[V][8];
        float sum = 0.0f, along = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int count = live ? min(a.cols - (t + T * i) * 8, 8) : 0;
            kind_values<KIND, CODES>(dr[i], g[i], a.f);
            kind_values<KIND, CODES>(zr[i], xhat[i], a.f);
            if constexpr (!kHold) load_weight<KIND>(a.gamma, (t + T * i) * 8, count, 1.0f, w[0], a.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xhat[i][j] = j < count ? (xhat[i][j] - centre) * scale : 0.0f;
                dw[i][j] = fmaf(g[i][j], xhat[i][j], dw[i][j]);
                db[i][j] += g[i][j];
                g[i][j] *= w[kHold ? i : 0][j];
                sum += g[i][j];
                along = fmaf(g[i][j], xhat[i][j], along);
            }
        }
        if (kAhead && base + step < a.rows) fetch(row + step);
        const float m0 = row_sum<T>(sum, shared) * n, m1 = row_sum<T>(along, shared) * n;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int gi = t + T * i, col = gi * 8, count = live ? min(a.cols - col, 8) : 0;
            if (count > 0) {
                float d[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = scale * (g[i][j] - m0 - xhat[i][j] * m1);
                if (a.dx) {
                    float e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] = d[j];
                    if (a.drop.rng) drop8(e, static_cast<uint64_t>(row) * blocks + gi, key, a.drop);
                    kind_store<KIND, OUT>(a.dx, row * a.lddx + col, count, e, a.round, a.f);
                }
                kind_store<KIND, OUT>(a.dz, row * a.lddz + col, count, d, a.round, a.f);
            }
        }
        if (!kAhead && base + step < a.rows) fetch(row + step);
    }
    if (!a.partial) return;
    float *record = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float (&s)[8] = which ? db[i] : dw[i];
            if constexpr (kRows > 1) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) joined[mine][8 * t + j] = s[j];
                __syncthreads();
                for (int c = threadIdx.x; c < kWidth; c += kThreads) {
                    float v = 0.0f;
#pragma unroll
                    for (int r = 0; r < kRows; ++r) v += joined[r][c];
                    if (kWidth * i + c < a.cols) record[which * a.cols + kWidth * i + c] = v;
                }
            } else {
                const int col = (t + T * i) * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < a.cols) record[which * a.cols + col + j] = s[j];
            }
        }
    }
}

// dgamma and dbeta from the workgroups' records: 32 columns per workgroup, 32 threads share a column's records, eight of them on their way at
// a time (with 16 threads and one at a time the addition of 1024 records took 20 us).
constexpr int kParamCols = 32, kParamThreads = 32;
__global__ __launch_bounds__(kParamCols *kParamThreads) void norm_param_kernel(const float *partial, int records, int cols, float *dgamma,
                                                                               float *dbeta)
{
    __shared__ float part[kParamThreads][kParamCols];
    const int in = threadIdx.x % kParamCols, c = blockIdx.x * kParamCols + in, lane = threadIdx.x / kParamCols, width = 2 * cols;
    float s = 0.0f;
    if (c < width)
        for (int r0 = lane; r0 < records; r0 += 8 * kParamThreads) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r0 + i * kParamThreads < records ? partial[static_cast<int64_t>(r0 + i * kParamThreads) * width + c] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
    part[lane][in] = s;
    __syncthreads();
    if (lane == 0 && c < width) {
#pragma unroll
        for (int r = 1; r < kParamThreads; ++r) s += part[r][in];
        if (c < cols) dgamma[c] = s;
        else dbeta[c - cols] = s;
    }
}

}  // namespace

int launch_layernorm_bwd(const LayerNorm &n, const void *dy, int64_t lddy, const void *z, int64_t ldz, const float *mean,
                         const float *rstd, const float *gamma, void *dz, int64_t lddz, void *dx, int64_t lddx, float *dgamma,
                         float *dbeta, const ElemFormat &f, hipStream_t stream)
{
    int cus = 0;
    int rc = device_cu_count(&cus);
    if (rc != FMT_OK) return rc;
    NormBwd a{dy, z, mean, rstd, gamma, dz, dx, nullptr, n.rows, lddy, ldz, lddz, lddx, static_cast<int32_t>(n.cols),
              n.result != FMT_RESULT_F32, make_drop(n.drop), f};
    int records = 0;
    with_shape(n.cols, [&](auto threads, auto eights) {
        constexpr int T = decltype(threads)::value, V = decltype(eights)::value, kThreads = kNormThreads<T>;
        const int64_t want = (n.rows + kThreads / T - 1) / (kThreads / T), most = cus;
        records = static_cast<int>(want < most ? want : most);
        if (records == 0) return;
        if (dgamma) {
            rc = get_acc_scratch(stream, static_cast<size_t>(records) * 2 * static_cast<size_t>(n.cols) * sizeof(float), &a.partial);
            if (rc != FMT_OK) return;
        }
        with_kind(f, n.store, n.result, [&](auto kind, auto in, auto out) {
            norm_bwd_kernel<T, V, decltype(kind)::value, decltype(in)::value, decltype(out)::value>
                <<<dim3(static_cast<uint32_t>(records)), dim3(kThreads), 0, stream>>>(a);
        });
    });
    if (rc != FMT_OK) return rc;
    if (dgamma)
        norm_param_kernel<<<dim3(static_cast<uint32_t>((2 * n.cols + kParamCols - 1) / kParamCols)), dim3(kParamCols * kParamThreads), 0, stream>>>(
            a.partial, records, static_cast<int>(n.cols), dgamma, dbeta);
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
