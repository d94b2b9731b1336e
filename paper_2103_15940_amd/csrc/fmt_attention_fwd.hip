// Attention, forward: the choice of kernels, and what joins parts of a row's keys.
#include <algorithm>

#include "fmt_attention_fwd.h"

namespace fmt {

extern template void run_attention_fwd<2>(const AttnFwd &, const FwdChoice &, dim3, hipStream_t);
extern template void run_attention_fwd<4>(const AttnFwd &, const FwdChoice &, dim3, hipStream_t);

namespace {

// Parts of a row's keys leave their maximum and sum apart, not the lse: that, rounded, would put 2^-22 of its size into every weight.
//
// Joins the parts of a row where they are few: a thread takes four columns, and reads all parts' records and columns at once (a wave per row,
// which waited for one after the other, took 10 us for 14000 rows).
constexpr int kJoinFew = 8;
__global__ __launch_bounds__(256) void attn_join_few_kernel(AttnFwd a)
{
    const AttnShape &s = a.s;
    const int fours = (s.dim + 3) / 4;
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (n >= all_rows * fours) return;
    const int64_t at = n / fours;
    const int col = static_cast<int>(n % fours) * 4, count = min(s.dim - col, 4);
    const float *tops = a.part + a.splits * all_rows * s.dim + at, *sums = tops + a.splits * all_rows;
    f32x4 o[kJoinFew];
    float l[kJoinFew], part_sum[kJoinFew], top = -INFINITY, sum = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kJoinFew; ++i) {
        const bool there = i < a.splits;
        l[i] = there ? tops[i * all_rows] : -INFINITY;
        part_sum[i] = there ? sums[i * all_rows] : 0.0f;
        o[i] = load4(a.part + (i * all_rows + at) * s.dim + col, there ? count : 0);
    }
#pragma unroll
    for (int i = 0; i < kJoinFew; ++i) top = fmaxf(top, l[i]);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < kJoinFew; ++i) {
        const float w = part_sum[i] * exp2_fast(l[i] - base);
        sum += w;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(w, o[i][j], v[j]);
    }
    const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= over;
    const int t = static_cast<int>(at % s.q_len), head = static_cast<int>(at / s.q_len % s.heads), b = static_cast<int>(at / s.q_len / s.heads);
    store4(const_cast<void *>(a.o.p), b * a.o.sb + t * a.o.st + head * a.o.sh + col, count, v, a.result, a.f);
    if (col == 0 && a.lse) a.lse[at] = lse_of(top, sum);
}

// And where they are many, a workgroup per row: first all parts' weights, then 8 or 16 threads per column with 8 parts each on their way.
constexpr int kJoinMost = 2048, kJoinThreads = 1024, kJoinWaves = kJoinThreads / 64;
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttnFwd a)
{
    __shared__ float weights[kJoinMost], outs[kJoinThreads], wave_tops[kJoinWaves], wave_sums[kJoinWaves];
    const AttnShape &s = a.s;
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, at = blockIdx.x;
    const float *tops = a.part + a.splits * all_rows * s.dim + at, *sums = tops + a.splits * all_rows;
    float top = -INFINITY, sum = 0.0f;
    for (int n = threadIdx.x; n < a.splits; n += kJoinThreads) top = fmaxf(top, weights[n] = tops[n * all_rows]);
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    if ((threadIdx.x & 63) == 0) wave_tops[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) top = fmaxf(top, wave_tops[w]);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int n = threadIdx.x; n < a.splits; n += kJoinThreads) sum += weights[n] = sums[n * all_rows] * exp2_fast(weights[n] - base);
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) sum += __shfl_xor(sum, w);
    if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) sum += wave_sums[w];
    const int width = s.dim <= 64 ? 64 : 128, groups = kJoinThreads / width, c = threadIdx.x % width, g = threadIdx.x / width;
    float o = 0.0f;
    if (c < s.dim) {
        const float *part = a.part + at * s.dim + c;
        for (int n0 = g; n0 < a.splits; n0 += 8 * groups) {
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = n0 + i * groups < a.splits ? part[(n0 + i * groups) * all_rows * s.dim] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) o = fmaf(n0 + i * groups < a.splits ? weights[n0 + i * groups] : 0.0f, p[i], o);
        }
    }
    outs[threadIdx.x] = o;
    __syncthreads();
    if (g != 0 || c >= s.dim) return;
    for (int i = 1; i < groups; ++i) o += outs[c + i * width];
    o = sum == 0.0f ? 0.0f : o / sum;
    const int t = static_cast<int>(at % s.q_len), head = static_cast<int>(at / s.q_len % s.heads), b = static_cast<int>(at / s.q_len / s.heads);
    const float v[4] = {o, 0.0f, 0.0f, 0.0f};
    store4(const_cast<void *>(a.o.p), b * a.o.sb + t * a.o.st + head * a.o.sh + c, 1, v, a.result, a.f);
    if (c == 0 && a.lse) a.lse[at] = lse_of(top, sum);
}

int launch_join(const AttnFwd &a, hipStream_t stream)
{
    const int64_t all_rows = static_cast<int64_t>(a.s.batch) * a.s.heads * a.s.q_len, fours = (a.s.dim + 3) / 4;
    if (a.splits > 1 && a.splits <= kJoinFew)
        attn_join_few_kernel<<<dim3(static_cast<uint32_t>((all_rows * fours + 255) / 256)), dim3(256), 0, stream>>>(a);
    else if (a.splits > 1)
        attn_join_kernel<<<dim3(static_cast<uint32_t>(all_rows)), dim3(kJoinThreads), 0, stream>>>(a);
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace

int launch_attention_fwd(const AttnShape &s, const AttnView &q, const AttnView &k, const AttnView &v, const AttnView &o, float *lse,
                         int32_t store, int32_t result, const ElemFormat &f, fmt_format_t fmt, hipStream_t stream)
{
    int cus = 0;
    int rc = device_cu_count(&cus);
    if (rc != FMT_OK) return rc;
    const bool few = static_cast<int64_t>(s.q_len) * s.group <= kFewRows;
    const int64_t row_tiles = few ? 1 : (static_cast<int64_t>(s.q_len) * s.group + kFwdRows - 1) / kFwdRows;
    // few rows, long keys: their keys in parts of four tiles or more, until the compute units have a workgroup each, or in the kernel for
    // few rows, which waits for memory, as many as they hold at a time (one more would be a second round for all of them)
    const int64_t work = row_tiles * s.kv_heads * s.batch, tile = few ? attention_few_tile(s.q_len * s.group, s.dim, store) : kFwdKeys, key_tiles = (s.k_len + tile - 1) / tile;
    const int64_t held = static_cast<int64_t>(cus) * (s.q_len * s.group <= 1 ? 4 : s.q_len * s.group <= 4 ? 3 : 2);
    int64_t splits = few ? held / work : (cus + work - 1) / work;
    if (splits > kJoinMost) splits = kJoinMost;
    if (splits > key_tiles / 4) splits = key_tiles / 4;
    if (splits < 1) splits = 1;
    const bool half = attention_half(fmt, s), check = fmt.e > 5;
    AttnFwd a{s, q, k, v, o, lse, result, static_cast<int32_t>(splits), nullptr, check ? kHalfUp : 1.0f, static_cast<int32_t>(row_tiles),
              store == FMT_STORE_CODE16, make_half_codes(fmt, s, store), f};
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, grid = work * splits;
    if (grid > most_workgroups(256)) {                     // in two calls
        if (s.batch == 1) return FMT_ERR_SHAPE;
        const int32_t first = s.batch / 2;
        const int64_t in = store == FMT_STORE_CODE16 ? 2 : 4, out = result == FMT_RESULT_CODE16 ? 2 : 4;
        rc = launch_attention_fwd(attn_from(s, 0, first), q, k, v, o, lse, store, result, f, fmt, stream);
        if (rc != FMT_OK) return rc;
        return launch_attention_fwd(attn_from(s, first, s.batch - first), attn_from(q, first, in), attn_from(k, first, in), attn_from(v, first, in),
                                    attn_from(o, first, out), lse ? lse + static_cast<int64_t>(first) * s.heads * s.q_len : nullptr, store, result, f,
                                    fmt, stream);
    }
    if (splits > 1) {
        rc = get_acc_scratch(stream, static_cast<size_t>(splits * all_rows * (s.dim + 2)) * sizeof(float), &a.part);
        if (rc != FMT_OK) return rc;
    }
    if (few) {
        rc = launch_attention_few(s, q, k, v, o, lse, store, result, a.splits, a.part, f, fmt, stream);
        return rc != FMT_OK ? rc : launch_join(a, stream);
    }
    const FwdChoice choice{half, half_pieces(fmt, result) == 2, half_kind(fmt, store)};
    const dim3 blocks(static_cast<uint32_t>(grid));
    if (s.dim <= 64) run_attention_fwd<2>(a, choice, blocks, stream);
    else run_attention_fwd<4>(a, choice, blocks, stream);
    return launch_join(a, stream);
}

}  // namespace fmt
