// Dropout of a matrix (fmt_norm.h has the mathematics).  Bound by memory, and not far from the vector units' time for the generator:
// 30011 x 4097 in binary16 codes, 492 MB, 93 us or 5.3 TB/s (a large elementwise pass: 6.2, with 16-byte accesses that odd rows do not
// allow).  Loads and stores marked as used once gained nothing.
#include <algorithm>

#include "fmt_norm.h"

namespace fmt {

namespace {

constexpr int kDropThreads = 256, kDropRuns = 4;      // eights per thread

template <int KIND, bool CODES, bool OUT>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const void *x, int64_t ldx, void *y, int64_t ldy, int64_t rows,
                                                                int64_t cols, uint32_t blocks, uint64_t before, Drop d, bool round, ElemFormat f)
{
    // (before: eights of the launches before this one)
    const uint64_t total = static_cast<uint64_t>(rows) * blocks, first = before + static_cast<uint64_t>(blockIdx.x) * (kDropThreads * kDropRuns);
    const uint64_t row0 = first / blocks;
    const uint32_t at0 = static_cast<uint32_t>(first - row0 * blocks);
    RawEight<CODES> raw[kDropRuns];
    int64_t to[kDropRuns];
    int count[kDropRuns];
    const uint32_t past0 = at0 + threadIdx.x, over0 = past0 / blocks;
    uint32_t g = past0 - over0 * blocks;                  // the eight's place in its row
    int64_t xo = static_cast<int64_t>(row0 + over0) * ldx + static_cast<int64_t>(g) * 8, yo = static_cast<int64_t>(row0 + over0) * ldy + static_cast<int64_t>(g) * 8;
#pragma unroll
    for (int i = 0; i < kDropRuns; ++i) {
        const int64_t left = cols - static_cast<int64_t>(g) * 8;
        count[i] = first + threadIdx.x + kDropThreads * i < total ? static_cast<int>(left < 8 ? left : 8) : 0;
        to[i] = yo;
        raw[i] = raw_load<CODES>(x, xo, count[i]);
        // on by 256 eights: the vector units have no division, and multiply 64 bits in a dozen steps
        g += kDropThreads;
        xo += 8 * kDropThreads;
        yo += 8 * kDropThreads;
        if (blocks >= kDropThreads) {
            if (g >= blocks) {
                g -= blocks;
                xo += ldx - 8 * static_cast<int64_t>(blocks);
                yo += ldy - 8 * static_cast<int64_t>(blocks);
            }
        } else {
            const uint32_t over = g / blocks;
            g -= over * blocks;
            xo += over * (ldx - 8 * static_cast<int64_t>(blocks));
            yo += over * (ldy - 8 * static_cast<int64_t>(blocks));
        }
    }
    const DropKey key = drop_key(d);
#pragma unroll
    for (int i = 0; i < kDropRuns; ++i) {
        if (count[i] <= 0) break;
        float v[8];
        kind_values<KIND, CODES>(raw[i], v, f);
        drop8(v, first + threadIdx.x + kDropThreads * i, key, d);
        kind_store<KIND, OUT>(y, to[i], count[i], v, round, f);
    }
}

}  // namespace

int launch_dropout(const void *x, int64_t ldx, void *y, int64_t ldy, int64_t rows, int64_t cols, const fmt_dropout_t &d, int32_t store,
                   int32_t result, const ElemFormat &f, hipStream_t stream)
{
    Drop drop = make_drop(d);
    drop.rng = d.rng;
    const uint32_t blocks = static_cast<uint32_t>((cols + 7) / 8);
    const uint64_t total = static_cast<uint64_t>(rows) * blocks, each = kDropThreads * kDropRuns, most = most_workgroups(kDropThreads);
    with_kind(f, store, result, [&](auto kind, auto in, auto out) {
        for (uint64_t before = 0; before < total;) {
            const uint64_t grid = std::min((total - before + each - 1) / each, most);
            dropout_kernel<decltype(kind)::value, decltype(in)::value, decltype(out)::value>
                <<<dim3(static_cast<uint32_t>(grid)), dim3(kDropThreads), 0, stream>>>(x, ldx, y, ldy, rows, cols, blocks, before, drop,
                                                                                       result != FMT_RESULT_F32, f);
            before += grid * each;
        }
    });
    FMT_HIP_CHECK(hipGetLastError());
    return FMT_OK;
}

}  // namespace fmt
