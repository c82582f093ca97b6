// GraphSAGE mean aggregation over one block (paper Eq. 16) whose source rows are held in 8 bits with scales:
//   out[i, c] = (1/n_i) sum over the edges e of row i of scale[indices[e], c / group] q[indices[e], c]
// What bounds the aggregation is the traffic of its input rows, random rows read once per edge; 8 bits are half of fp16's.
//
// 16 columns, 16 bytes, are a lane's; a row's lanes are the smallest power of two that covers it, up to a wavefront (wider rows:
// slabs of 1,024 columns, a share of the grid each), and the wavefront's groups of lanes take the entries of an output row in
// turn, kFlight of each under way at a time.  Their sums, 32 bits each, are joined by exchanges between lanes: the order depends
// on the row's own entries and the call's width alone, so the result is reproducible bit for bit.
#include <algorithm>

#include "common.h"
#include "layer_types.h"

namespace mqg {

namespace {

constexpr int kCols = 16;             // columns of a lane
constexpr int kFlight = 4;

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

template <typename T, int QTYPE, int LANES>
__global__ void __launch_bounds__(kBlock)
k_mean_aggregate_q8(MeanQ8Args a) {
    constexpr int G = kWave / LANES;  // entries side by side
    const int lane = lane_id() % LANES, g = lane_id() / LANES;
    const uint32_t slab = blockIdx.x / a.row_blocks, row_block = blockIdx.x - slab * a.row_blocks;
    const int col0 = (static_cast<int>(slab) * LANES + lane) * kCols;
    const bool live = col0 < a.dim, whole = col0 + kCols <= a.dim;
    const int at = live ? col0 : 0;
    const int scale_at = a.group ? at / a.group : 0;
    const int64_t n = a.sizes[0] < a.cap_dst ? a.sizes[0] : a.cap_dst;
    const int64_t step = int64_t(a.row_blocks) * kWavesPerBlock;
    for (int64_t i = int64_t(row_block) * kWavesPerBlock + (threadIdx.x >> 6); i < n; i += step) {
        const int b = a.indptr[i], e = a.indptr[i + 1];
        float acc[kCols];
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
        for (int p0 = b; p0 < e; p0 += kFlight * G) {
            int64_t r[kFlight];
            float sc[kFlight];
            Words4 w[kFlight];
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                const int p = p0 + u * G + g;
                r[u] = a.indices[p < e ? p : e - 1];       // past the end: the last entry again, not added
            }
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                const uint8_t *row = a.q + r[u] * a.q_stride + at;
                sc[u] = a.scale[r[u] * a.scale_stride + scale_at];
                if (whole || !live) {
                    w[u] = whole ? *reinterpret_cast<const AnyWords4 *>(row) : Words4{0, 0, 0, 0};
                } else {                                   // the row's last columns, byte by byte: nothing outside the row is read
                    w[u] = Words4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
                        if (col0 + j < a.dim) w[u][j / 4] |= static_cast<uint32_t>(row[j]) << (8 * (j % 4));
                }
            }
#pragma unroll
            for (int u = 0; u < kFlight; ++u)
                if (p0 + u * G + g < e) add_scaled<QTYPE>(acc, w[u], sc[u]);
        }
#pragma unroll
        for (int off = LANES; off < kWave; off <<= 1)
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[j] += __shfl_xor(acc[j], off, kWave);
        if (g != 0 || !live) continue;
        const float count = e > b ? static_cast<float>(e - b) : 1.f;
        T *out = static_cast<T *>(a.out) + i * a.out_stride;
        constexpr int V = Vec<T>::kLen;
#pragma unroll
        for (int k = 0; k < kCols / V; ++k) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = acc[k * V + j] / count;
            store_vec(out, col0 / V + k, a.dim, v);
        }
    }
}

template <typename T, int QTYPE>
int launch_mean_q8(mqg_ctx *ctx, MeanQ8Args a, hipStream_t s) {
    const int lanes_needed = static_cast<int>(ceil_div(a.dim, kCols));
    const int64_t slabs = ceil_div(lanes_needed, kWave);
    // (a launch has fewer than 2^32 threads)
    a.row_blocks = static_cast<uint32_t>(std::min<int64_t>(ceil_div(a.cap_dst, kWavesPerBlock), std::max<int64_t>(1, std::min<int64_t>(256 * 32, (int64_t(1) << 23) / slabs))));
    const int grid = static_cast<int>(a.row_blocks * slabs);
#define MQG_GO(L) MQG_LAUNCH(ctx, "k_mean_aggregate_q8", s, (k_mean_aggregate_q8<T, QTYPE, L><<<grid, kBlock, 0, s>>>(a)))
    if (lanes_needed <= 1) MQG_GO(1);
    else if (lanes_needed <= 2) MQG_GO(2);
    else if (lanes_needed <= 4) MQG_GO(4);
    else if (lanes_needed <= 8) MQG_GO(8);
    else if (lanes_needed <= 16) MQG_GO(16);
    else if (lanes_needed <= 32) MQG_GO(32);
    else MQG_GO(64);
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
