// GraphSAGE mean aggregation over one block (paper Eq. 16) whose source rows are held in 8 bits with scales:
//   out[i, c] = (1/n_i) sum over the edges e of row i of scale[indices[e], c / group] q[indices[e], c]
// What bounds it is memory: the lines of 128 bytes that its input rows lie in, as often as an entry meets them, and the lookups of their scales.  4.4 M entries
// of 256 columns out of 1.35 M rows take 239 us, 184 of them (6.2 TB/s of row lines, what an elementwise kernel reaches) without the scales' loads; 2.8 M entries of 128 columns
// 85, 70 without.  8 bits are half of fp16's lines: the same entries of fp16 rows take k_mean_aggregate 359 and 115 us.
//
// 16 columns, 16 bytes, are a lane's; an output row is the work of the smallest power of two of lanes that covers it, up to a wavefront (wider rows:
// slabs of 1,024 columns, a share of the grid each), so that no sum crosses lanes: the order depends on the row's own entries alone, and the result is
// reproducible bit for bit.  Eight input rows are on their way at a time.  (Measured before: a wavefront to an output row, its groups of lanes taking the entries
// in turn and joining their sums: 295,000 rows of 5 entries and 100 columns 320 us, 95 now; 10,200 of 25 and 602 98 and 34; 16 instead of eight rows on their way 38.)
#include <algorithm>

#include "common.h"
#include "layer_types.h"

namespace mqg {

namespace {

constexpr int kCols = 16;             // columns of a lane

struct MeanQ8Args {
    const int32_t *indptr, *indices;
    const int64_t *sizes;
    const uint8_t *q;
    const float *scale;
    void *out;
    int64_t q_stride, scale_stride, out_stride, cap_dst;
    int32_t dim, group;               // group: columns per scale, 0 = the row
    uint32_t row_blocks;              // workgroups per slab
};

typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef Words4 AnyWords4 __attribute__((aligned(1)));

template <int QTYPE>
__device__ __forceinline__ void add_scaled(float (&acc)[kCols], Words4 w, float scale) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (QTYPE == MQG_Q_E4M3) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[k]), false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[k]), true);
            acc[4 * k] += scale * lo[0];
            acc[4 * k + 1] += scale * lo[1];
            acc[4 * k + 2] += scale * hi[0];
            acc[4 * k + 3] += scale * hi[1];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[4 * k + j] += scale * static_cast<float>(static_cast<int8_t>(w[k] >> (8 * j)));
        }
    }
}

typedef int32_t Index4 __attribute__((ext_vector_type(4)));
typedef Index4 AnyIndex4 __attribute__((aligned(4)));

template <typename T, int QTYPE, int LANES>
__global__ void __launch_bounds__(kBlock)
k_mean_aggregate_q8(MeanQ8Args a) {
    constexpr int kRows = kBlock / LANES;
    const int lane = static_cast<int>(threadIdx.x) % LANES;
    const uint32_t slab = blockIdx.x / a.row_blocks, row_block = blockIdx.x - slab * a.row_blocks;
    const int col0 = (static_cast<int>(slab) * LANES + lane) * kCols;
    if (col0 >= a.dim) return;
    // The last lane of a row whose columns are not a multiple of 16 takes the row's last 16, nothing outside the row is read: those that it shares with
    // the lane before come out the same, unless a group of scales ends among them; then, and in rows of fewer than 16, it stores its own alone.
    const bool narrow = a.dim < kCols;
    const int at = narrow ? 0 : col0 + kCols <= a.dim ? col0 : a.dim - kCols;
    const int scale_at = a.group ? (at + kCols - 1) / a.group : 0;
    const int own = narrow || (a.group && at / a.group != scale_at) ? col0 : at;     // the first column that it stores
    const int64_t n = a.sizes[0] < a.cap_dst ? a.sizes[0] : a.cap_dst;
    const uint8_t *q = a.q + at;
    const float *scale = a.scale + (narrow ? 0 : scale_at);
    for (int64_t i = int64_t(row_block) * kRows + threadIdx.x / LANES; i < n; i += int64_t(a.row_blocks) * kRows) {
        const int b = a.indptr[i], e = a.indptr[i + 1];
        float acc[kCols];
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
        // N entries from p on: all their loads, then their additions; past the row's end the last one again, times 0
        auto batch = [&](int p, auto number) __attribute__((always_inline)) {
            constexpr int N = decltype(number)::value;
            int64_t r[N];
            float sc[N];
            Words4 w[N];
            if (p + N <= e) {
#pragma unroll
                for (int u = 0; u < N; u += 4) {
                    const Index4 x = *reinterpret_cast<const AnyIndex4 *>(a.indices + p + u);
#pragma unroll
                    for (int k = 0; k < 4; ++k) r[u + k] = x[k];
                }
            } else {
#pragma unroll
                for (int u = 0; u < N; ++u) r[u] = a.indices[p + u < e ? p + u : e - 1];
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                sc[u] = scale[r[u] * a.scale_stride];
                if (!narrow) {
                    w[u] = *reinterpret_cast<const AnyWords4 *>(q + r[u] * a.q_stride);
                } else {
                    w[u] = Words4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < kCols - 1; ++j)
                        if (j < a.dim) w[u][j / 4] |= static_cast<uint32_t>(q[r[u] * a.q_stride + j]) << (8 * (j % 4));
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) add_scaled<QTYPE>(acc, w[u], p + u < e ? sc[u] : 0.f);
        };
        int p = b;
        for (; e - p > 4; p += 8) batch(p, std::integral_constant<int, 8>());
        if (e - p > 0) batch(p, std::integral_constant<int, 4>());
        const float count = e > b ? static_cast<float>(e - b) : 1.f, inv = 1.f / count;
        T *out = static_cast<T *>(a.out) + i * a.out_stride;
#pragma unroll
        for (int j = 0; j < kCols; ++j) {                  // the quotient by the reciprocal, and its remainder's, which infinity has none of
            const float quot = acc[j] * inv, whole = fmaf(fmaf(-quot, count, acc[j]), inv, quot);
            acc[j] = fabsf(quot) < __uint_as_float(0x7F800000u) ? whole : quot;
        }
        if (own == at && !narrow) {
            constexpr int V = Vec<T>::kLen;
#pragma unroll
            for (int k = 0; k < kCols / V; ++k) {
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = acc[k * V + j];
                store_vec(out + at, k, kCols, v);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kCols; ++j)
                if (at + j >= own && at + j < a.dim) out[at + j] = static_cast<T>(acc[j]);
        }
    }
}

template <typename T, int QTYPE>
int launch_mean_q8(mqg_ctx *ctx, MeanQ8Args a, hipStream_t s) {
    const int lanes_needed = static_cast<int>(ceil_div(a.dim, kCols));
    int lanes = 1;
    while (lanes < lanes_needed && lanes < kWave) lanes <<= 1;
    const int64_t slabs = ceil_div(lanes_needed, kWave);
    // (a launch has fewer than 2^32 threads)
    const int64_t most = std::max<int64_t>(1, (int64_t(1) << 23) / slabs);
    a.row_blocks = static_cast<uint32_t>(std::min<int64_t>(ceil_div(a.cap_dst, kBlock / lanes), most));
    const int grid = static_cast<int>(a.row_blocks * slabs);
#define MQG_GO(L) MQG_LAUNCH(ctx, "k_mean_aggregate_q8", s, (k_mean_aggregate_q8<T, QTYPE, L><<<grid, kBlock, 0, s>>>(a)))
    switch (lanes) {
        case 1: MQG_GO(1); break;
        case 2: MQG_GO(2); break;
        case 4: MQG_GO(4); break;
        case 8: MQG_GO(8); break;
        case 16: MQG_GO(16); break;
        case 32: MQG_GO(32); break;
        default: MQG_GO(64);
    }
#undef MQG_GO
    return MQG_OK;
}

template <typename T>
int launch_mean_q8_of(mqg_ctx *ctx, const MeanQ8Args &a, int32_t q_type, hipStream_t s) {
    return q_type == MQG_Q_E4M3 ? launch_mean_q8<T, MQG_Q_E4M3>(ctx, a, s) : launch_mean_q8<T, MQG_Q_INT8>(ctx, a, s);
}

}  // namespace

int run_mean_aggregate_q8(mqg_ctx *ctx, const mqg_block *b, const void *q, int64_t q_stride, int32_t q_type, int32_t group, const float *scale,
                          int64_t scale_stride, void *out, int64_t out_stride, int32_t dim, int32_t dtype, hipStream_t s) {
    if (b->cap_dst == 0) return MQG_OK;
    const MeanQ8Args a{b->indptr, b->indices, b->sizes, static_cast<const uint8_t *>(q), scale, out, q_stride, scale_stride, out_stride,
                       b->cap_dst, dim, group, 1};
    if (dtype == MQG_F16) return launch_mean_q8_of<F16>(ctx, a, q_type, s);
    if (dtype == MQG_BF16) return launch_mean_q8_of<BF16>(ctx, a, q_type, s);
    return launch_mean_q8_of<float>(ctx, a, q_type, s);
}

}  // namespace mqg
