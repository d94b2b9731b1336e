// Attention, forward: the kernels (fmt_attention.h has the mathematics and the layouts), compiled per head size in
// fmt_attention_fwd_64.hip and fmt_attention_fwd_128.hip.
#pragma once

#include "fmt_attention.h"

namespace fmt {

struct AttnFwd {
    AttnShape s;
    AttnView q, k, v, o;
    float *lse;               // [batch][heads][q_len]
    int32_t result;
    int32_t splits;           // parts of a row's keys
    float *part;              // splits > 1: [splits][batch * heads * q_len][dim] normalised outputs, then as many maxima in base 2, then sums
    float up;                 // what the fp16 operands are multiplied by
    int32_t row_tiles;
    bool codes;               // how q, k and v are stored
    HalfCodes hc;
    ElemFormat f;
};

constexpr int kFwdRows = 128, kFwdKeys = 64;

struct FwdBlock {
    uint32_t id;
    int b, kh, split, row0;
};

// Workgroups of a causal mask differ in their keys, and with two to a compute unit, of which an XCD has 32, its workgroups n and n + 32 meet
// in one: the second 32 go in reverse, so that long ones meet short ones (binary16, 8 heads of 128: 2 x 4096 tokens 170 -> 139 us, 8 x 1024
// 50 -> 41, 1 x 8192 265 -> 250; of 64: 2 x 4096 111 -> 85).  Where there are more, the later ones go where there is room, and a turn gained
// nothing (16 heads of 64: 162 -> 169).
__device__ __forceinline__ uint32_t fwd_order(const AttnFwd &a, uint32_t i, uint32_t n)
{
    constexpr uint32_t kUnits = 32;
    const uint32_t at = i >> 3, mine = (n >> 3) + ((i & 7) < (n & 7) ? 1 : 0);
    const bool turn = a.s.causal && at >= kUnits && mine <= 2 * kUnits;
    return xcd_order(i, n) - at + (turn ? kUnits + mine - 1 - at : at);
}

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
__device__ __forceinline__ void fwd_store(const AttnFwd &a, const f32x16 (&o)[DT], int split, int b, int t, int head, int half, float over, float top, float sum)
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
    if (part) {
        float *records = a.part + a.splits * all_rows * s.dim + split * all_rows + at;
        records[0] = top;
        records[a.splits * all_rows] = sum;
    } else if (a.lse) {
        a.lse[at] = lse_of(top, sum);
    }
}

// A workgroup takes 128 rows of one (batch, kv head), a wave 32 of them: S^T = K Q^T gives every lane one row's scores, half of them each for
// lanes l and l + 32, so the running maximum and sum of a row need one exchange per tile of 64 keys.
// What a launch of the kernels of one head size (DT blocks of 32 columns) needs to know beside their arguments.
struct FwdChoice {
    bool half, two;           // fp16 operands, in one or two pieces of P
    int kind;                 // kHalfCodes and so on
};
template <int DT>
void run_attention_fwd(const AttnFwd &a, const FwdChoice &c, dim3 blocks, hipStream_t stream);

namespace {

template <int DT>
struct FwdShared {
    AttnTile<kPieces, DT, kFwdKeys> ks, vs;
};

template <int DT>
__device__ __forceinline__ void fwd_pieces(const AttnFwd &a, uint32_t id, FwdShared<DT> &sh)
{
    constexpr int NQ = kPieces, NP = kProbPieces;
    AttnTile<kPieces, DT, kFwdKeys> &ks = sh.ks, &vs = sh.vs;
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
    if (live) fwd_store<DT>(a, o, split, b, t, head, half, over, top, sum);
}

template <int DT>
__global__ __launch_bounds__(256) void attn_fwd_kernel(AttnFwd a)
{
    __shared__ FwdShared<DT> sh;
    fwd_pieces<DT>(a, fwd_order(a, blockIdx.x, gridDim.x), sh);
}

// The same on operands of one fp16 value each, P in NP pieces of fp16.  The next tile's elements are on their way from memory while a
// tile is computed; they are rounded and converted on their way into the other of two LDS buffers, so a tile costs one barrier.
//
// Measured: 16384 tokens, 8 heads over 2, head size 128, window 2048 and 16 sinks in binary16: 211 to 231 us, 560 to 610 TFLOP/s of S and O
// (with both pieces of P 840 to 920; a large product reaches 1282).  The matrix cores are busy for 50 % of the time, LDS for 42 % (two fifths of that bank
// conflicts), and between the two products lie exponentials, conversions and sums, at two workgroups per compute unit.
// What V lost to fp16 is added after the tiles: with one channel of 2^-30, so that every tile has some, the call takes 2.3 times as long, and computed again
// with pieces of bf16 3.2 times (4096 tokens, 8 heads of 128, 1/6/9: 267, 617, 858 us).
// Short sequences (32 x 128 tokens, 12 heads of 64) are a chain of two tiles: 18 us against 7 for their bytes.
template <int NP, int DT, int KIND>
__global__ __launch_bounds__(256, DT == 2 ? (half_is_codes(KIND) ? 3 : 2) : (half_is_codes(KIND) ? 2 : 1)) void attn_fwd_half_kernel(AttnFwd a)
{
    __shared__ union Shared {
        struct {
            AttnTile<1, DT, kFwdKeys> ks[2], vs[2];
        } half;
        FwdShared<DT> pieces;
        uint32_t cuts[4];
        __device__ Shared() {}
    } sh;
    auto &ks = sh.half.ks, &vs = sh.half.vs;
    constexpr int kEights = 4 * DT, kLoads = kFwdKeys * kEights / 256;
    constexpr bool CODES = half_is_codes(KIND);
    const AttnShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const FwdBlock blk = fwd_block(a, fwd_order(a, blockIdx.x, gridDim.x));
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

    const AttnTiles tiles = attn_tiles(s, seq.length, i0, i1, kFwdKeys);
    const int count = tiles.count();
    const int begin = static_cast<int>(static_cast<int64_t>(count) * split / a.splits);
    const int end = static_cast<int>(static_cast<int64_t>(count) * (split + 1) / a.splits);
    RawEight<CODES> kr[kLoads], vr[kLoads];
    const int key_in = threadIdx.x / kEights, col_in = (threadIdx.x % kEights) * 8;     // + 256 / kEights keys per load
    constexpr int kStep = 256 / kEights, kSize = CODES ? 2 : 4;
    const char *kp = static_cast<const char *>(a.k.p) + (b * a.k.sb + kh * a.k.sh + key_in * a.k.st + col_in) * kSize;
    const char *vp = static_cast<const char *>(a.v.p) + (b * a.v.sb + kh * a.v.sh + key_in * a.v.st + col_in) * kSize;
    const int64_t kst = a.k.st * kSize, vst = a.v.st * kSize;
    auto fetch = [&](int n) __attribute__((always_inline)) {
        const int k0 = tiles.at(n) * kFwdKeys;
        const char *kt = kp + k0 * kst, *vt = vp + k0 * vst;
        if (s.dim == 32 * DT && k0 + kFwdKeys <= seq.length) {           // nothing is missing: no lane asks
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                kr[i] = raw_load<CODES>(kt + i * kStep * kst, 0, 8);
                vr[i] = raw_load<CODES>(vt + i * kStep * vst, 0, 8);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int have = k0 + key_in + i * kStep < seq.length ? s.dim - col_in : 0;
                kr[i] = raw_load<CODES>(kt + i * kStep * kst, 0, have);
                vr[i] = raw_load<CODES>(vt + i * kStep * vst, 0, have);
            }
        }
    };
    if (begin < end) fetch(begin);

    bool ignore = false;
    u32x4 q[2 * DT];
#pragma unroll
    for (int kk = 0; kk < 2 * DT; ++kk) {
        const int col = 16 * kk + 8 * half;
        q[kk] = half_signed(
            raw_half<KIND, false>(raw_load<CODES>(a.q.p, b * a.q.sb + t * a.q.st + head * a.q.sh + col, live ? s.dim - col : 0), a.up, a.hc, high, ignore, a.f),
            s.scale);
    }
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;
    const float scale2 = s.scale == 0.0f ? 1.0f : fabsf(s.scale2) / (a.up * a.up);
    const AttnKeys sees = attn_keys(s, seq.length, pos);
    constexpr bool kCuts = half_has_limit(KIND);
    uint32_t cuts = 0;                                     // which 32nds of the tiles lost bits of V
    const int cut_tiles = (end - begin + 31) / 32;
    for (int n = begin; n < end; ++n) {
        const int k0 = tiles.at(n) * kFwdKeys, buf = (n - begin) & 1;
        bool cut = false;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int key = key_in + i * (256 / kEights);
            *reinterpret_cast<u32x4 *>(&ks[buf].e[0][key][col_in]) = raw_half<KIND, false>(kr[i], a.up, a.hc, high, ignore, a.f);
            *reinterpret_cast<u32x4 *>(&vs[buf].e[0][key][col_in]) = raw_half<KIND, kCuts>(vr[i], a.up, a.hc, high_value, cut, a.f);
        }
        if constexpr (kCuts) {
            if (__any(cut)) cuts |= 1u << ((n - begin) / cut_tiles);
        }
        __syncthreads();
        if (n + 1 < end) fetch(n + 1);
        f32x16 x[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[0][i] = x[1][i] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 2 * DT; ++kk)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {              // two sums in turn: a product does not wait for the one before it
                u32x4 f[1];
                read_rows(ks[buf], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                x[kt] = mfma_f16(f[0], q[kk], x[kt]);
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
        if (__any(high_score > top + kFwdSlack)) {
            const float next = fmaxf(top, high_score);
            const float shrink = next == -INFINITY ? 1.0f : exp2_fast(top - next);
            top = next;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
        }
        const float base = (top == -INFINITY ? 0.0f : top) - kFwdUp;
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
    if (kCuts && a.up != 1.0f) {
        bool pieces = half_flag<CODES>(high, high_value, a.hc);
        if (lane == 0) sh.cuts[wave] = cuts;
        __syncthreads();
        cuts = __builtin_amdgcn_readfirstlane(sh.cuts[0] | sh.cuts[1] | sh.cuts[2] | sh.cuts[3]);      // the same in the whole workgroup
        __syncthreads();
        if (__builtin_expect(cuts && !pieces, 0)) {
            // what was cut, over the tiles that it may be in, with the weights relative to the rows' largest scores
            bool lost = false;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= kRestUp;
            const float base = (top == -INFINITY ? 0.0f : top) - kFwdUp;
#pragma unroll 1
            for (int n = begin; n < end; ++n) {
                if (!(cuts >> ((n - begin) / cut_tiles) & 1u)) continue;
                fetch(n);
                const int k0 = tiles.at(n) * kFwdKeys;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int key = key_in + i * kStep;
                    float v[8];
                    raw_values(vr[i], v, a.f);
                    *reinterpret_cast<u32x4 *>(&ks[0].e[0][key][col_in]) = raw_half<KIND, false>(kr[i], a.up, a.hc, high, ignore, a.f);
                    *reinterpret_cast<u32x4 *>(&vs[0].e[0][key][col_in]) = half_rest(v, a.up, lost);
                }
                __syncthreads();
#pragma unroll 1
                for (int kt = 0; kt < 2; ++kt) {
                    f32x16 x;
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
                    for (int kk = 0; kk < 2 * DT; ++kk) {
                        u32x4 f[1];
                        read_rows(ks[0], 32 * kt + (lane & 31), 16 * kk + 8 * half, f);
                        x = mfma_f16(f[0], q[kk], x);
                    }
                    attn_hide(sees, k0 + 32 * kt + 4 * half, x);
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) {
                        float p[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) p[j] = exp2_fast(fmaf(x[8 * kb + j], scale2, -base));
                        u32x4 pp[NP];
                        f16_pieces<NP>(p, pp);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            u32x4 f[1];
                            read_columns(vs[0], 32 * kt + 16 * kb, 32 * d, lane, f);
#pragma unroll
                            for (int w = NP - 1; w >= 0; --w) o[d] = mfma_f16(f[0], pp[w], o[d]);
                        }
                    }
                }
                __syncthreads();
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= 1.0f / kRestUp;
            pieces = __syncthreads_or(lost);
        }
        if (__builtin_expect(pieces, 0)) {
            fwd_pieces<DT>(a, blk.id, sh.pieces);
            return;
        }
    }
    sum += __shfl_xor(sum, 32);
    const float over = sum == 0.0f ? 0.0f : 1.0f / (sum * a.up);
    // (the sum without P's factor: its logarithm would have fewer bits)
    if (live) fwd_store<DT>(a, o, split, b, t, head, half, over, top, sum * exp2_fast(-kFwdUp));
}

}  // namespace

template <int DT>
void run_attention_fwd(const AttnFwd &a, const FwdChoice &c, dim3 blocks, hipStream_t stream)
{
    if (!c.half) {
        attn_fwd_kernel<DT><<<blocks, dim3(256), 0, stream>>>(a);
        return;
    }
    auto go = [&](auto kind) {
        if (c.two) attn_fwd_half_kernel<2, DT, decltype(kind)::value><<<blocks, dim3(256), 0, stream>>>(a);
        else attn_fwd_half_kernel<1, DT, decltype(kind)::value><<<blocks, dim3(256), 0, stream>>>(a);
    };
    switch (c.kind) {
    case kHalfCodes: go(std::integral_constant<int, kHalfCodes>{}); break;
    case kHalfFloat: go(std::integral_constant<int, kHalfFloat>{}); break;
    case kBf16Codes: go(std::integral_constant<int, kBf16Codes>{}); break;
    case kSixCodes: go(std::integral_constant<int, kSixCodes>{}); break;
    case kOtherCodes: go(std::integral_constant<int, kOtherCodes>{}); break;
    case kMagicFloat: go(std::integral_constant<int, kMagicFloat>{}); break;
    default: go(std::integral_constant<int, kIntegerFloat>{}); break;
    }
}

}  // namespace fmt
