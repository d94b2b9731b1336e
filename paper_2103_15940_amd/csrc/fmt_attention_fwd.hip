// Attention, forward: the choice of kernels, and what joins parts of a row's keys.
#include <algorithm>

#include "fmt_attention_fwd.h"

namespace fmt {

extern template void run_attention_fwd<2>(const AttnFwd &, const FwdChoice &, dim3, hipStream_t);
extern template void run_attention_fwd<4>(const AttnFwd &, const FwdChoice &, dim3, hipStream_t);

namespace {

// Joins the parts of a row, a workgroup per row: each of its four waves takes every fourth part, a lane two columns.
__global__ __launch_bounds__(256) void attn_join_kernel(AttnFwd a)
{
    __shared__ float outs[4][128], sums[4], tops[4];
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, at = blockIdx.x;
    const float *lse = a.part + a.splits * all_rows * s.dim + at;
    float top = -INFINITY;
    for (int n = threadIdx.x; n < a.splits; n += 256) top = fmaxf(top, lse[n * all_rows]);
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, o[2] = {0.0f, 0.0f};
#pragma unroll 4
    for (int n = wave; n < a.splits; n += 4) {
        const float w = exp2_fast(lse[n * all_rows] - base);
        const float *part = a.part + (n * all_rows + at) * s.dim;
        sum += w;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (lane + 64 * j < s.dim) o[j] = fmaf(w, part[lane + 64 * j], o[j]);
    }
    if (lane == 0) sums[wave] = sum;
    outs[wave][lane] = o[0];
    outs[wave][lane + 64] = o[1];
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= s.dim) return;
    sum = sums[0] + sums[1] + sums[2] + sums[3];
    const float out = sum == 0.0f ? 0.0f : (outs[0][c] + outs[1][c] + outs[2][c] + outs[3][c]) / sum;
    const int t = static_cast<int>(at % s.q_len), head = static_cast<int>(at / s.q_len % s.heads), b = static_cast<int>(at / s.q_len / s.heads);
    const float v[4] = {out, 0.0f, 0.0f, 0.0f};
    store4(const_cast<void *>(a.o.p), b * a.o.sb + t * a.o.st + head * a.o.sh + c, 1, v, a.result, a.f);
    if (c == 0 && a.lse) a.lse[at] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
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
    // few rows, long keys: their keys in parts of four tiles or more, until the compute units have a workgroup each (four of the kernel for
    // few rows, whose workgroups wait for memory)
    const int64_t work = row_tiles * s.kv_heads * s.batch, tile = few ? attention_few_tile(s.dim, store) : kFwdKeys, key_tiles = (s.k_len + tile - 1) / tile;
    const int64_t want = few ? 4 * cus : cus;
    int64_t splits = work >= want ? 1 : (want + work - 1) / work;
    if (splits > key_tiles / 4) splits = key_tiles / 4;
    if (splits < 1) splits = 1;
    const bool half = attention_half(fmt), check = fmt.e > 5;
    AttnFwd a{s, q, k, v, o, lse, result, static_cast<int32_t>(splits), nullptr, check ? kHalfUp : 1.0f, static_cast<int32_t>(row_tiles),
              store == FMT_STORE_CODE16, make_half_codes(fmt, f), f};
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, grid = work * splits;
    if (grid > 0x7FFFFFFF) return FMT_ERR_SHAPE;
    if (splits > 1) {
        rc = get_acc_scratch(stream, static_cast<size_t>(splits * all_rows * (s.dim + 1)) * sizeof(float), &a.part);
        if (rc != FMT_OK) return rc;
    }
    if (few) {
        rc = launch_attention_few(s, q, k, v, o, lse, store, result, a.splits, a.part, f, fmt, stream);
        if (rc != FMT_OK) return rc;
        if (splits > 1) attn_join_kernel<<<dim3(static_cast<uint32_t>(all_rows)), dim3(256), 0, stream>>>(a);
        FMT_HIP_CHECK(hipGetLastError());
        return FMT_OK;
    }
    const FwdChoice choice{half, half_pieces(fmt, result) == 2, a.codes, check};
    const dim3 blocks(static_cast<uint32_t>(grid));
    if (s.dim <= 64) run_attention_fwd<2>(a, choice, blocks, stream);
    else run_attention_fwd<4>(a, choice, blocks, stream);
    if (splits > 1) attn_join_kernel<<<dim3(static_cast<uint32_t>(all_rows)), dim3(256), 0, stream>>>(a);
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
