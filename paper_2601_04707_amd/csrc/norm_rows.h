// What the norms of rows have in common (norm.hip, layer_norm.hip): how a row is laid out over lanes, rows outside 32 bits' range, the output in 8 bits, and
// the sum of the workgroups' shares of a gradient.
#pragma once

#include "common.h"
#include "layer_types.h"

namespace mqg {
namespace {

constexpr int kNormParts = 512;      // workgroups of the root-mean-square norm's backward at most

__device__ __forceinline__ int64_t rows_of(const int64_t *num_rows, int64_t cap) {
    if (!num_rows) return cap;
    const int64_t n = *num_rows;
    return n < cap ? (n > 0 ? n : 0) : cap;
}

// The mean of squares and eps of a row outside this range: its sums may have lost terms at either end of 32 bits' range, and so may the square of the factor
// R = 1/sqrt(mean).  They are taken again of s times a power of two, row_unit, after which they are well inside (large: |s| up to 2^128 becomes up to 2^56, sums
// up to 2^126; small, where eps doesn't make up for the lost terms: 2^-149 to 2^-43 become 2^-59 to 2^47).  Rows of fp16 never need it but for zeros.
// The comparison costs the others nothing to 1.5 % (300,000 x 100 fp32 66.9 -> 67.8 us).
__device__ __forceinline__ bool odd_mean(float mean) {
    return __float_as_uint(mean) - __float_as_uint(0x1p-100f) > __float_as_uint(0x1p+100f) - __float_as_uint(0x1p-100f);
}
__device__ __forceinline__ float row_unit(float mean) { return mean > 0x1p+100f ? 0x1p-72f : mean < 0x1p-100f ? 0x1p+90f : 1.f; }
// The mean of s times unit, or infinity, whose factor is 0, where the row's own factor, unit times as large, is above 32 bits' numbers: zeros without an epsilon,
// and rows whose root mean square is below 2^-128.
__device__ __forceinline__ float unit_mean(float squares, int dim, float eps, float unit) {
    const float mean = squares / static_cast<float>(dim) + eps * unit * unit;
    return sqrtf(mean) < unit * 0x1p-128f ? __uint_as_float(0x7F800000u) : mean;
}
// What is the same in all lanes of a wavefront, for the compiler, too: scalar registers
template <int LANES>
__device__ __forceinline__ float of_wave(float v) {
    return LANES < kWave ? v : __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

// V values of a row in 8 bits
template <int V, typename S>
__device__ __forceinline__ void store_q(uint8_t *row, const Span<V> &at, int dim, const float (&z)[V], const S &s, int q_type) {
    uint32_t w[V / 4];
    to_8bit(z, s, q_type, w);
    if (at.skip == 0 && dim >= V) {
        typedef uint32_t Words __attribute__((ext_vector_type(V / 4)));
        typedef Words AnyWords __attribute__((aligned(1)));
        Words v;
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            if constexpr (V == 4) v = w[k];
            else v[k] = w[k];
        }
        *reinterpret_cast<AnyWords *>(row + at.base) = v;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (at.mine(j) && at.base + j < dim) row[at.base + j] = static_cast<uint8_t>(w[j / 4] >> (8 * (j % 4)));
    }
}

// out[c] = sum over the parts, from column `split` on out2[c - split], 16 columns a workgroup: 64 threads take a column's parts in turn, eight of them on their way together, and their sums are
// added in order.
constexpr int kSumCols = 16, kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
k_sum_parts(const float *__restrict__ parts, int num_parts, int dim, float *__restrict__ out, int split, float *__restrict__ out2) {
    constexpr int kTurns = kSumThreads / kSumCols, kAhead = 8;
    __shared__ float lds[kTurns][kSumCols + 1];
    const int c = static_cast<int>(blockIdx.x) * kSumCols + static_cast<int>(threadIdx.x) % kSumCols;
    const int turn = static_cast<int>(threadIdx.x) / kSumCols;
    float v = 0.f;
    if (c < dim)
        for (int p0 = turn; p0 < num_parts; p0 += kAhead * kTurns) {
            float x[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) x[k] = p0 + k * kTurns < num_parts ? parts[int64_t(p0 + k * kTurns) * dim + c] : 0.f;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) v += x[k];
        }
    lds[turn][threadIdx.x % kSumCols] = v;
    __syncthreads();
    // the 64 sums of a column by the lanes of a wavefront
    const int col = static_cast<int>(threadIdx.x) / kWave;
    v = lanes_sum(lds[lane_id()][col], kWave);
    const int to = static_cast<int>(blockIdx.x) * kSumCols + col;
    if (lane_id() == 0 && to < dim) *(to < split ? out + to : out2 + (to - split)) = v;
}
static_assert(kSumThreads / kSumCols == kWave && kSumThreads / kWave == kSumCols, "a wavefront adds a column");

// How a row is laid out: lanes, and vectors per lane.  As few lanes as hold it with up to four vectors each within a wavefront; longer rows have a
// workgroup of 512 (8,192 rows of 8,192 bf16: 109 us and the backward 112; 256 lanes 144 and 112, 1,024 126 and 120), the longest one of 1,024.
// Few rows are spread as wide as they go: there is nothing else to do.
struct RowShape {
    int lanes, nv;
};
constexpr int kFewRows = 256;
RowShape row_shape(int dim, int vec, int64_t rows) {
    const int vecs = static_cast<int>(ceil_div(dim, vec));
    for (int lanes = 4; lanes <= kWave; lanes <<= 1)
        if (vecs <= lanes) return {lanes, 1};
    if (rows <= kFewRows) {
        if (vecs <= 256) return {256, 1};
        if (vecs > 512 && vecs <= 1024) return {1024, 1};
    }
    if (vecs <= 4 * kWave) return {kWave, static_cast<int>(ceil_div(vecs, kWave))};
    if (vecs <= 2 * 512) return {512, static_cast<int>(ceil_div(vecs, 512))};
    return {1024, vecs <= 2 * 1024 ? 2 : 4};
}

#define MQG_NORM_SHAPES(T, GO)                                     \
    switch (sh.lanes) {                                            \
        case 4: GO(T, 4, 1); break;                                \
        case 8: GO(T, 8, 1); break;                                \
        case 16: GO(T, 16, 1); break;                              \
        case 32: GO(T, 32, 1); break;                              \
        case 64:                                                   \
            if (sh.nv == 1) GO(T, 64, 1);                          \
            else if (sh.nv == 2) GO(T, 64, 2);                     \
            else if (sh.nv == 3) GO(T, 64, 3);                     \
            else GO(T, 64, 4);                                     \
            break;                                                 \
        case 256: GO(T, 256, 1); break;                            \
        case 512:                                                  \
            if (sh.nv == 1) GO(T, 512, 1);                         \
            else GO(T, 512, 2);                                    \
            break;                                                 \
        default:                                                   \
            if (sh.nv == 1) GO(T, 1024, 1);                        \
            else if (sh.nv == 2) GO(T, 1024, 2);                   \
            else if constexpr (sizeof(T) == 4) GO(T, 1024, 4);     \
    }

// A call that moves twice what the chip's memory-side cache holds leaves little of its own output there: that goes past the caches (109,000 x 602
// fp32 rows, four times 262 MB: 202 -> 190 us; 295,000 x 256 bf16, four times 151 MB: 112 -> 97; backward of these 194 -> 191 and 111 -> 108).  Smaller ones
// keep it for the next reader, though they would be faster by themselves, too (40,000 x 1,000 bf16, 320 MB: 55 -> 49; 60,000 x 256 fp32 42 -> 37).
constexpr int64_t kPastBytes = int64_t(512) << 20;

}  // namespace
}  // namespace mqg
