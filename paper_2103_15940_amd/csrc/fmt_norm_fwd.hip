// Dropout, residual and layer norm, forward (fmt_norm.h has the mathematics).
//
// A row stays in the registers of its threads, 8 columns each and piece.  All of a row's loads, weights among them, are on their way
// before the first is used: a wave has one row, so its time is one trip to memory, two reductions and the stores.
//
// Measured: 4096 x 1024 in bfloat16 with residual and dropout 14 us (33.6 MB: 5.4 at the rate of a large elementwise pass): all 1024 workgroups
// are on the card at once, so reads, generator and writes come one after the other for all of them.  128 x 128 in 1/6/9, fp32: 5.2 us, 32 x 1024:
// 6.5, the chain alone.
#include <algorithm>

#include "fmt_norm.h"

namespace fmt {

namespace {

struct NormFwd {
    const void *x, *res;
    const float *gamma, *beta;
    void *z, *y;
    float *mean, *rstd;
    int64_t rows, ldx, ldres, ldz, ldy;
    int64_t first;            // row of the launch's first
    int32_t cols;
    float eps;
    bool round;               // whether fp32 results are rounded
    Drop drop;
    ElemFormat f;
};

template <int T>
constexpr int kNormThreads = T < 256 ? 256 : T;

template <int T, int V, int KIND, bool CODES, bool OUT>
__global__ __launch_bounds__(kNormThreads<T>) void norm_fwd_kernel(NormFwd a)
{
    __shared__ float shared[T > 64 ? kNormThreads<T> / 64 : 1];
    constexpr int kRows = kNormThreads<T> / T;
    constexpr bool kEarly = V <= 2;                       // registers for the weights as well
    const int t = threadIdx.x % T;
    const int64_t row = a.first + static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / T;
    const bool live = row < a.rows;                       // no early exit: lanes of one wave add up together
    const int blocks = (a.cols + 7) >> 3;
    RawEight<CODES> xr[V], rr[V];
    RawEight<false> wr[kEarly ? V : 1], br[kEarly ? V : 1];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int col = (t + T * i) * 8, count = live ? a.cols - col : 0;
        xr[i] = raw_load<CODES>(a.x, row * a.ldx + col, count);
        if (a.res) rr[i] = raw_load<CODES>(a.res, row * a.ldres + col, count);
        if constexpr (kEarly) {
            if (a.gamma) wr[i] = raw_load<false>(a.gamma, col, count);
            if (a.beta) br[i] = raw_load<false>(a.beta, col, count);
        }
    }
    float z[V][8];
    float sum = 0.0f;
    DropKey key{};
    if (a.drop.rng) key = drop_key(a.drop);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = t + T * i, col = g * 8;
        const int count = live ? min(a.cols - col, 8) : 0;
        kind_values<KIND, CODES>(xr[i], z[i], a.f);
        if (a.drop.rng) drop8(z[i], static_cast<uint64_t>(row) * blocks + g, key, a.drop);
        if (a.res) {
            float r[8];
            kind_values<KIND, CODES>(rr[i], r, a.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[i][j] = __fadd_rn(r[j], z[i][j]);
        }
        if (a.res || a.drop.rng) round_kind<KIND>(z[i], a.f);       // (what lies past the last column is 0 and stays it)
        if (a.z && count > 0) kind_store<KIND, OUT, true>(a.z, row * a.ldz + col, count, z[i], false, a.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += z[i][j];
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
            if constexpr (kEarly) {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.0f, b[j] = 0.0f;
                if (a.gamma) kind_values<KIND, false>(wr[i], w, a.f);
                if (a.beta) kind_values<KIND, false>(br[i], b, a.f);
            } else {
                load_weight<KIND>(a.gamma, col, count, 1.0f, w, a.f);
                load_weight<KIND>(a.beta, col, count, 0.0f, b, a.f);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = fmaf((z[i][j] - mean) * rstd, w[j], b[j]);
            kind_store<KIND, OUT>(a.y, row * a.ldy + col, count, y, a.round, a.f);
        }
    }
}

}  // namespace

int launch_layernorm_fwd(const LayerNorm &n, const void *x, int64_t ldx, const void *res, int64_t ldres, const float *gamma,
                         const float *beta, float eps, void *z, int64_t ldz, void *y, int64_t ldy, float *mean, float *rstd,
                         const ElemFormat &f, hipStream_t stream)
{
    NormFwd a{x, res, gamma, beta, z, y, mean, rstd, n.rows, ldx, ldres, ldz, ldy, 0, static_cast<int32_t>(n.cols), eps,
              n.result != FMT_RESULT_F32, make_drop(n.drop), f};
    with_shape(n.cols, [&](auto threads, auto eights) {
        constexpr int T = decltype(threads)::value, V = decltype(eights)::value, kThreads = kNormThreads<T>, kRows = kThreads / T;
        with_kind(f, n.store, n.result, [&](auto kind, auto in, auto out) {
            for (int64_t left; (left = n.rows - a.first) > 0;) {
                const int64_t grid = std::min((left + kRows - 1) / kRows, most_workgroups(kThreads));
                norm_fwd_kernel<T, V, decltype(kind)::value, decltype(in)::value, decltype(out)::value>
                    <<<dim3(static_cast<uint32_t>(grid)), dim3(kThreads), 0, stream>>>(a);
                a.first += grid * kRows;
            }
        });
    });
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
