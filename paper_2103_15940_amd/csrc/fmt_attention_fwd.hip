// Attention, forward (fmt_attention.h has the mathematics and the layouts).
#include <algorithm>
#include <type_traits>

#include "fmt_attention.h"

namespace fmt {

namespace {

struct AttnFwd {
    AttnShape s;
    AttnView q, k, v, o;
    float *lse;               // [batch][heads][q_len]
    int32_t result;
    int32_t splits;           // parts of a row's keys
    float *part;              // splits > 1: [splits][batch * heads * q_len][dim] normalised outputs, then as many lse in base 2
    uint32_t *flags;          // per workgroup: whether it is left to the pieces of bf16; or nullptr
    float up;                 // what the fp16 operands are multiplied by
    int32_t row_tiles;
    uint32_t blocks;          // workgroups of the first launch
    bool codes;               // how q, k and v are stored
    HalfCodes hc;
    ElemFormat f;
};

constexpr int kFwdRows = 128, kFwdKeys = 64;

struct FwdBlock {
    uint32_t id;
    int b, kh, split, row0;
};

// Which rows a workgroup takes.  The later ones of a causal mask see more keys: they go first.
__device__ __forceinline__ FwdBlock fwd_block(const AttnFwd &a, uint32_t id)
{
    const uint32_t tile = id % a.row_tiles, rest = id / a.row_tiles;
    const uint32_t kh = rest % a.s.kv_heads, rest2 = rest / a.s.kv_heads;
    return FwdBlock{id, static_cast<int>(rest2 / a.splits), static_cast<int>(kh), static_cast<int>(rest2 % a.splits),
                    static_cast<int>(a.s.causal ? a.row_tiles - 1 - tile : tile) * kFwdRows};
}

// A lane's outputs: its row of a wave's results, over its sum.
template <int DT>
__device__ __forceinline__ void fwd_store(const AttnFwd &a, const f32x16 (&o)[DT], int split, int b, int t, int head, int half, float over, float lse2)
{
    const AttnShape &s = a.s;
    const int64_t at = (static_cast<int64_t>(b) * s.heads + head) * s.q_len + t;
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len;
    const bool part = a.splits > 1;
    void *out = part ? static_cast<void *>(a.part) : const_cast<void *>(a.o.p);
    const int64_t base = part ? (split * all_rows + at) * s.dim : b * a.o.sb + t * a.o.st + head * a.o.sh;
    const int result = part ? FMT_RESULT_F32 : a.result;
    store_row<DT>(out, base, half, s.dim, o, over, result, a.f);
    if (half != 0) return;
    if (part) a.part[a.splits * all_rows * s.dim + split * all_rows + at] = lse2;
    else if (a.lse) a.lse[at] = lse2 * 0.6931471805599453f;
}

// A workgroup takes 128 rows of one (batch, kv head), a wave 32 of them: S^T = K Q^T gives every lane one row's scores, half of them each for
// lanes l and l + 32, so the running maximum and sum of a row need one exchange per tile of 64 keys.
template <int DT>
__device__ __forceinline__ void fwd_pieces(const AttnFwd &a, uint32_t id, AttnTile<kPieces, DT, kFwdKeys> &ks, AttnTile<kPieces, DT, kFwdKeys> &vs)
{
    constexpr int NQ = kPieces, NP = kProbPieces;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const FwdBlock blk = fwd_block(a, id);
    const int b = blk.b, split = blk.split, kh = blk.kh;
    const AttnSeq seq = attn_seq(s, b);
    const int rows = s.q_len * s.group;
    const int row0 = blk.row0, row = row0 + wave * 32 + (lane & 31);
    const int t = row / s.group, head = kh * s.group + row % s.group;
    const bool live = row < rows;
    const int pos = seq.first + t;
    const int64_t i0 = static_cast<int64_t>(seq.first) + row0 / s.group;
    const int64_t i1 = static_cast<int64_t>(seq.first) + (min(row0 + kFwdRows, rows) - 1) / s.group;

    u32x4 q[2 * DT][NQ];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half, count = live ? min(s.dim - col, 8) : 0;
        float v[8];
        if (count > 0) {
            load8_any(a.q.p, b * a.q.sb + t * a.q.st + head * a.q.sh + col, count, v, a.codes, a.f);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        }
        bf16_pieces<NQ>(v, q[kk]);
    }

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;
    const int64_t kbase = b * a.k.sb + kh * a.k.sh, vbase = b * a.v.sb + kh * a.v.sh;
    const AttnTiles tiles = attn_tiles(s, seq.length, i0, i1, kFwdKeys);
    const int count = tiles.count();
    const int begin = static_cast<int>(static_cast<int64_t>(count) * split / a.splits);
    const int end = static_cast<int>(static_cast<int64_t>(count) * (split + 1) / a.splits);
    for (int n = begin; n < end; ++n) {
        const int k0 = tiles.at(n) * kFwdKeys;
        __syncthreads();
        load_tokens<NQ, DT, kFwdKeys>(ks, a.k.p, kbase, a.k.st, k0, seq.length, s.dim, a.codes, a.f);
        load_tokens<NQ, DT, kFwdKeys>(vs, a.v.p, vbase, a.v.st, k0, seq.length, s.dim, a.codes, a.f);
        __syncthreads();
        f32x16 x[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kt][i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                u32x4 f[NQ];
                read_rows(ks, 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                x[kt] = mfma_pieces<NQ, NQ>(f, q[kk], x[kt]);
            }
        }
        const bool all = attn_sees_all(s, seq.length, i0, i1, k0, k0 + kFwdKeys);
        float high = top;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float y = x[kt][i] * s.scale2;
                if (!all && !attn_sees(s, seq.length, pos, k0 + 32 * kt + 8 * (i / 4) + 4 * half + (i & 3))) y = -INFINITY;
                x[kt][i] = y;
                high = fmaxf(high, y);
            }
        high = fmaxf(high, __shfl_xor(high, 32));
        const float base = high == -INFINITY ? 0.0f : high, shrink = exp2_fast(top - base);
        top = high;
        sum *= shrink;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = exp2_fast(x[kt][8 * kb + j] - base);
                    sum += p[j];
                }
                u32x4 pp[NP];
                bf16_pieces<NP>(p, pp);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[NQ];
                    read_columns(vs, 32 * kt + 16 * kb, 32 * d, lane, f);
                    o[d] = mfma_pieces<NQ, NP>(f, pp, o[d]);
                }
            }
    }
    sum += __shfl_xor(sum, 32);
    const float over = sum == 0.0f ? 0.0f : 1.0f / sum;          // a row that sees nothing: 0
    if (live) fwd_store<DT>(a, o, split, b, t, head, half, over, sum == 0.0f ? -INFINITY : top + log2f(sum));
}

// All workgroups of a launch (no flags), or those that the launch before has flagged, among few that stay.
template <int DT>
__global__ __launch_bounds__(256) void attn_fwd_kernel(AttnFwd a)
{
    __shared__ AttnTile<kPieces, DT, kFwdKeys> ks, vs;
    for (uint32_t i = blockIdx.x; i < a.blocks; i += gridDim.x) {
        const uint32_t id = xcd_order(i, a.blocks);
        if (a.flags == nullptr || a.flags[id] != 0) fwd_pieces<DT>(a, id, ks, vs);       // (the same in the whole workgroup)
    }
}

// The same on operands of one fp16 value each, P in NP pieces of fp16.  The next tile's elements are on their way from memory while a
// tile is computed; they are rounded and converted on their way into the other of two LDS buffers, so a tile costs one barrier.
template <int NP, int DT, bool CODES>
__global__ __launch_bounds__(256, CODES || DT == 2 ? 2 : 1) void attn_fwd_half_kernel(AttnFwd a)
{
    __shared__ AttnTile<1, DT, kFwdKeys> ks[2], vs[2];
    constexpr int kEights = 4 * DT, kLoads = kFwdKeys * kEights / 256;
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const FwdBlock blk = fwd_block(a, xcd_order(blockIdx.x, gridDim.x));
    const int b = blk.b, split = blk.split, kh = blk.kh;
    const AttnSeq seq = attn_seq(s, b);
    const int rows = s.q_len * s.group;
    const int row0 = blk.row0, row = row0 + wave * 32 + (lane & 31);
    const int t = row / s.group, head = kh * s.group + row % s.group;
    const bool live = row < rows;
    const int pos = seq.first + t;
    const int64_t i0 = static_cast<int64_t>(seq.first) + row0 / s.group;
    const int64_t i1 = static_cast<int64_t>(seq.first) + (min(row0 + kFwdRows, rows) - 1) / s.group;
    uint32_t high = 0, high_value = 0;

    const int64_t kbase = b * a.k.sb + kh * a.k.sh, vbase = b * a.v.sb + kh * a.v.sh;
    const AttnTiles tiles = attn_tiles(s, seq.length, i0, i1, kFwdKeys);
    const int count = tiles.count();
    const int begin = static_cast<int>(static_cast<int64_t>(count) * split / a.splits);
    const int end = static_cast<int>(static_cast<int64_t>(count) * (split + 1) / a.splits);
    RawEight<CODES> kr[kLoads], vr[kLoads];
    const int key_in = threadIdx.x / kEights, col_in = (threadIdx.x % kEights) * 8;     // + 256 / kEights keys per load
    auto fetch = [&](int n) __attribute__((always_inline)) {
        const int k0 = tiles.at(n) * kFwdKeys;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int key = k0 + key_in + i * (256 / kEights);
            const int have = key < seq.length ? s.dim - col_in : 0;
            kr[i] = raw_load<CODES>(a.k.p, kbase + key * a.k.st + col_in, have);
            vr[i] = raw_load<CODES>(a.v.p, vbase + key * a.v.st + col_in, have);
        }
    };
    if (begin < end) fetch(begin);

    u32x4 q[2 * DT];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half;
        q[kk] = half_signed(
            raw_half<CODES>(raw_load<CODES>(a.q.p, b * a.q.sb + t * a.q.st + head * a.q.sh + col, live ? s.dim - col : 0), a.up, a.hc, high, a.f), s.scale);
    }
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;
    const float scale2 = s.scale == 0.0f ? 1.0f : fabsf(s.scale2) / (a.up * a.up);
    const AttnKeys sees = attn_keys(s, seq.length, pos);
    for (int n = begin; n < end; ++n) {
        const int k0 = tiles.at(n) * kFwdKeys, buf = (n - begin) & 1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int key = key_in + i * (256 / kEights);
            *reinterpret_cast<u32x4 *>(&ks[buf].e[0][key][col_in]) = raw_half<CODES>(kr[i], a.up, a.hc, high, a.f);
            *reinterpret_cast<u32x4 *>(&vs[buf].e[0][key][col_in]) = raw_half<CODES>(vr[i], a.up, a.hc, high_value, a.f);
        }
        __syncthreads();
        if (n + 1 < end) fetch(n + 1);
        f32x16 x[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kt][i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < 2 * DT; ++kk) {
                u32x4 f[1];
                read_rows(ks[buf], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                x[kt] = mfma_f16(f[0], q[kk], x[kt]);
            }
        }
        if (!attn_sees_all(s, seq.length, i0, i1, k0, k0 + kFwdKeys)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) attn_hide(sees, k0 + 32 * kt + 4 * half, x[kt]);
        }
        float high_score = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) high_score = fmaxf(high_score, x[kt][i]);
        high_score = fmaxf(high_score, __shfl_xor(high_score, 32)) * scale2;
        if (__any(high_score > top)) {                    // else the running maximum stays in all of the wave's rows
            const float next = fmaxf(top, high_score);
            const float shrink = next == -INFINITY ? 1.0f : exp2_fast(top - next);
            top = next;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
        }
        const float base = (top == -INFINITY ? 0.0f : top) - kProbUp;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = exp2_fast(fmaf(x[kt][8 * kb + j], scale2, -base));
                    sum += p[j];
                }
                u32x4 pp[NP];
                f16_pieces<NP>(p, pp);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 f[1];
                    read_columns(vs[buf], 32 * kt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                    for (int w = NP - 1; w >= 0; --w) o[d] = mfma_f16(f[0], pp[w], o[d]);
                }
            }
    }
    sum += __shfl_xor(sum, 32);
    const float over = sum == 0.0f ? 0.0f : 1.0f / (sum * a.up);
    if (a.flags) {
        const bool flag = half_flag<CODES>(high, high_value, a.hc);
        if (threadIdx.x == 0) a.flags[blk.id] = flag;
    }
    if (live) fwd_store<DT>(a, o, split, b, t, head, half, over, sum == 0.0f ? -INFINITY : top - kProbUp + log2f(sum));
}

// Joins the parts of a row: one wave per row.
__global__ __launch_bounds__(256) void attn_join_kernel(AttnFwd a)
{
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63;
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (at >= all_rows) return;
    const float *lse = a.part + a.splits * all_rows * s.dim + at;
    float top = -INFINITY;
    for (int n = lane; n < a.splits; n += 64) top = fmaxf(top, lse[n * all_rows]);
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, o[2] = {0.0f, 0.0f};
    for (int n = 0; n < a.splits; ++n) {
        const float w = exp2_fast(lse[n * all_rows] - base);
        sum += w;
        const float *part = a.part + (n * all_rows + at) * s.dim;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (2 * lane + j < s.dim) o[j] = fmaf(w, part[2 * lane + j], o[j]);
    }
    const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int t = static_cast<int>(at % s.q_len), head = static_cast<int>(at / s.q_len % s.heads), b = static_cast<int>(at / s.q_len / s.heads);
    const float v[4] = {o[0] * over, o[1] * over, 0.0f, 0.0f};
    if (2 * lane < s.dim)
        store4(const_cast<void *>(a.o.p), b * a.o.sb + t * a.o.st + head * a.o.sh + 2 * lane, min(s.dim - 2 * lane, 2), v, a.result, a.f);
    if (lane == 0 && a.lse) a.lse[at] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace

int launch_attention_fwd(const AttnShape &s, const AttnView &q, const AttnView &k, const AttnView &v, const AttnView &o, float *lse,
                         int32_t store, int32_t result, const ElemFormat &f, fmt_format_t fmt, hipStream_t stream)
{
    int cus = 0;
    int rc = device_cu_count(&cus);
    if (rc != FMT_OK) return rc;
    const int64_t row_tiles = (static_cast<int64_t>(s.q_len) * s.group + kFwdRows - 1) / kFwdRows;
    // few rows, long keys: their keys in parts of four tiles or more, until the compute units have a workgroup each
    const int64_t work = row_tiles * s.kv_heads * s.batch, key_tiles = (s.k_len + kFwdKeys - 1) / kFwdKeys;
    int64_t splits = work >= cus ? 1 : (cus + work - 1) / work;
    if (splits > key_tiles / 4) splits = key_tiles / 4;
    if (splits < 1) splits = 1;
    AttnFwd a{s, q, k, v, o, lse, result, static_cast<int32_t>(splits), nullptr, nullptr, 1.0f, static_cast<int32_t>(row_tiles), 0, false, make_half_codes(fmt, f), f};
    const int64_t all_rows = static_cast<int64_t>(s.batch) * s.heads * s.q_len, grid = work * splits;
    if (grid > 0x7FFFFFFF) return FMT_ERR_SHAPE;
    const bool half = attention_half(fmt), flagged = half && fmt.e > 5;
    const size_t part = splits > 1 ? static_cast<size_t>(splits * all_rows * (s.dim + 1)) : 0, flags = flagged ? static_cast<size_t>(grid) : 0;
    if (part + flags) {
        float *scratch = nullptr;
        rc = get_acc_scratch(stream, (part + flags) * sizeof(float), &scratch);
        if (rc != FMT_OK) return rc;
        if (part) a.part = scratch;
        if (flagged) a.flags = reinterpret_cast<uint32_t *>(scratch + part);
    }
    a.blocks = static_cast<uint32_t>(grid);
    a.codes = store == FMT_STORE_CODE16;
    with_dim(s.dim, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (half) {
            a.up = flagged ? kHalfUp : 1.0f;
            const dim3 blocks(a.blocks), threads(256);
            const bool two = half_pieces(fmt, result) == 2;
            if (two && a.codes) attn_fwd_half_kernel<2, DT, true><<<blocks, threads, 0, stream>>>(a);
            else if (two) attn_fwd_half_kernel<2, DT, false><<<blocks, threads, 0, stream>>>(a);
            else if (a.codes) attn_fwd_half_kernel<1, DT, true><<<blocks, threads, 0, stream>>>(a);
            else attn_fwd_half_kernel<1, DT, false><<<blocks, threads, 0, stream>>>(a);
        }
        if (!half || flagged)
            attn_fwd_kernel<DT><<<dim3(flagged ? std::min(a.blocks, static_cast<uint32_t>(cus)) : a.blocks), dim3(256), 0, stream>>>(a);
    });
    if (splits > 1) attn_join_kernel<<<dim3(static_cast<uint32_t>((all_rows + 3) / 4)), dim3(256), 0, stream>>>(a);
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
