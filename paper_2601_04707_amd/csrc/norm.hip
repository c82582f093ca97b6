// Root-mean-square norm of the rows between two layers, with the residual's addition and an output in 8 bits, and its backward.
//
//   forward    s = x + r,  y = s rsqrt(mean(s^2) + eps) w,  8 bits: scale = max(max|y| / top, 2^-126) per row or group of columns,
//              q = y / scale rounded to nearest even (top = 448: e4m3, 127: int8)
//   backward   with R = rsqrt(mean(s^2) + eps) and c = R^2 mean(gy w s):  gx = R (gy w - c s) + gs,  gw = sum over rows of gy s R
//
// Both are bound by memory: every input is read once and every output written once, a row stays in registers in between.  A row
// is the work of 4 to 64 lanes of a wavefront, of 256, 512 or 1,024 threads, by its length, so that a reduction over a short row is a few exchanges between
// lanes and short rows fill the wavefront.  Measured, of the 6.2 TB/s that an elementwise kernel reads and writes at: forward 295,000 x 256 fp16 into e4m3
// 97 us = 5.4, 109,000 x 602 fp32 184 to 187 us = 5.6 to 5.7, 20,000 x 2,048 fp32 107 to 109 us = 6.0 to 6.1; backward 295,000 x 256 fp16 104 us = 5.8, 8,192 x 8,192 bf16 107 us = 5.0.  The
// last vector of a row is loaded without a branch (Span): element by element, backward rows of 250 fp16 columns took 227 us instead of 116, of 100 fp32 columns 412
// instead of 188, for the wait in that branch, which held up the row that was on its way.
#include <algorithm>

#include "common.h"
#include "norm_rows.h"

namespace mqg {

int64_t norm_scratch_bytes(int32_t dim) { return int64_t(kNormParts) * dim * int64_t(sizeof(float)); }

namespace {

struct NormArgs {
    const void *x, *residual;
    const float *weight;
    const int64_t *num_rows;
    void *sum, *y;
    uint8_t *q;
    float *scale;
    int64_t x_stride, residual_stride, sum_stride, y_stride, q_stride, scale_stride;
    int64_t cap_rows;
    float eps;
    int32_t dim, q_type, group;       // group: columns per scale, 0 = the row
};

// What the lanes of a row find together.  Rows of several wavefronts exchange through LDS: two buffers in turn, so that one barrier
// per exchange is enough (who writes a buffer again has passed the barrier behind which all have read it).
template <int LANES>
struct RowLanes {
    static constexpr int kWaves = LANES / kWave;
    float *lds;
    int turn = 0;
    __device__ __forceinline__ explicit RowLanes(float *l) : lds(l) {}
    template <typename F>
    __device__ __forceinline__ float join(float v, F f) {
        float *buf = lds + turn * kWaves;
        turn ^= 1;
        if (lane_id() == 0) buf[threadIdx.x >> 6] = v;
        __syncthreads();
        float all = buf[0];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) all = f(all, buf[k]);
        return all;
    }
    // two sums by one exchange (of buffers of twice the size; not with the others in one kernel)
    __device__ __forceinline__ void sum_both(float *x, float *y) {
        *x = lanes_sum(*x, LANES < kWave ? LANES : kWave);
        *y = lanes_sum(*y, LANES < kWave ? LANES : kWave);
        if constexpr (LANES > kWave) {
            float *buf = lds + turn * 2 * kWaves;
            turn ^= 1;
            if (lane_id() == 0) {
                buf[2 * (threadIdx.x >> 6)] = *x;
                buf[2 * (threadIdx.x >> 6) + 1] = *y;
            }
            __syncthreads();
            float u = 0.f, v = 0.f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                u += buf[2 * k];
                v += buf[2 * k + 1];
            }
            *x = u;
            *y = v;
        }
    }
    __device__ __forceinline__ float sum(float v) {
        v = lanes_sum(v, LANES < kWave ? LANES : kWave);
        if constexpr (LANES > kWave) v = join(v, [](float a, float b) { return a + b; });
        return v;
    }
    __device__ __forceinline__ uint32_t max(uint32_t v) {
        v = lanes_max(v, LANES < kWave ? LANES : kWave);
        if constexpr (LANES > kWave)
            v = __float_as_uint(join(__uint_as_float(v), [](float a, float b) { return __uint_as_float(max_u32(__float_as_uint(a), __float_as_uint(b))); }));
        return v;
    }
};

template <typename T, int LANES, int NV, bool PAST>
__global__ void __launch_bounds__(LANES > kBlock ? LANES : kBlock)
k_rms_norm(NormArgs a) {
    constexpr int V = Vec<T>::kLen;
    constexpr int kThreads = LANES > kBlock ? LANES : kBlock;
    constexpr int kRows = kThreads / LANES;                // rows of a workgroup
    __shared__ float lds[LANES > kWave ? 2 * (LANES / kWave) : 1];
    RowLanes<LANES> lanes(lds);
    const int lane = static_cast<int>(threadIdx.x) % LANES;
    const int64_t n = rows_of(a.num_rows, a.cap_rows);
    const int dim = a.dim;
    const float top = a.q_type == MQG_Q_E4M3 ? 448.f : 127.f;
    const int group_lanes = a.group / V;                   // lanes that share a scale, 0 = the row's
    const bool full = dim == LANES * NV * V;               // every lane's vectors are its own
    float w[NV][V];
    Span<V> at[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        at[k] = Span<V>(k * LANES + lane, dim);
        load_weight(a.weight, at[k], dim, w[k]);
    }
    for (int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES; row < n; row += int64_t(gridDim.x) * kRows) {
        using W = typename Vec<T>::Whole;
        W raw[NV], more[NV];
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *r0 = static_cast<const T *>(a.residual) + row * a.residual_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            raw[k] = load_span(x, at[k], dim);
            if (a.residual) more[k] = load_span(r0, at[k], dim);
        }
        float s[NV][V];
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[k][j] = static_cast<float>(raw[k][j]);
                if (a.residual) s[k][j] += static_cast<float>(more[k][j]);
            }
        if (!full) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (at[k].skip > 0)
#pragma unroll
                    for (int j = 0; j < V; ++j) s[k][j] = at[k].mine(j) ? s[k][j] : 0.f;
        }
        if (a.sum) {
            T *sum = static_cast<T *>(a.sum) + row * a.sum_stride;
#pragma unroll
            for (int k = 0; k < NV; ++k) store_span<PAST>(sum, at[k], dim, s[k]);
        }
        float squares = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float part = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) part += s[k][j] * s[k][j];
            squares += part;
        }
        float mean = of_wave<LANES>(lanes.sum(squares)) / static_cast<float>(dim) + a.eps;
        if (ballot64(odd_mean(mean))) {                    // (not of rows of several wavefronts: the same in all of them)
            const float unit = row_unit(mean);
            squares = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s[k][j] *= unit;
                    squares += s[k][j] * s[k][j];
                }
            mean = unit_mean(of_wave<LANES>(lanes.sum(squares)), dim, a.eps, unit);
        }
        const float r = 1.0f / sqrtf(mean);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s[k][j] *= w[k][j];
        if (a.y) {
            T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = s[k][j] * r;
                store_span<PAST>(y, at[k], dim, v);
            }
        }
        if (!a.q) continue;
        uint8_t *q = a.q + row * a.q_stride;
        float *scale = a.scale + row * a.scale_stride;
        if (!full) {                                       // (another lane's columns: zero times a weight that is not finite would be no number)
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (at[k].skip > 0)
#pragma unroll
                    for (int j = 0; j < V; ++j) s[k][j] = at[k].mine(j) ? s[k][j] : 0.f;
        }
        uint32_t most[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            most[k] = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) most[k] = max_u32(most[k], __float_as_uint(s[k][j]) & 0x7FFFFFFFu);
        }
        if (group_lanes == 0) {
            uint32_t m = most[0];
#pragma unroll
            for (int k = 1; k < NV; ++k) m = max_u32(m, most[k]);
            const Scale sc = scale_of(lanes.max(m), r, top);
            if (lane == 0) scale[0] = sc.scale;
#pragma unroll
            for (int k = 0; k < NV; ++k) store_q(q, at[k], dim, s[k], sc, a.q_type);
        } else {
            const int width = group_lanes < LANES ? group_lanes : LANES;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const Scale sc = scale_of(lanes_max(most[k], width), r, top);
                const int i = k * LANES + lane;
                if (lane % width == 0 && i * V < dim) scale[i / group_lanes] = sc.scale;
                store_q(q, at[k], dim, s[k], sc, a.q_type);
            }
        }
    }
}

struct NormGradArgs {
    const void *grad_y, *s, *grad_sum;
    const float *weight;
    const int64_t *num_rows;
    void *grad_x;
    float *parts;                     // [grid x dim] every workgroup's share of the weight's gradient; null if that is not wanted
    int64_t gy_stride, s_stride, gs_stride, gx_stride;
    int64_t cap_rows;
    float eps;
    int32_t dim;
};

template <typename T, int LANES, int NV, bool PAST>
__global__ void __launch_bounds__(LANES > kBlock ? LANES : kBlock)
k_rms_norm_backward(NormGradArgs a) {
    using W = typename Vec<T>::Whole;
    constexpr int V = Vec<T>::kLen;
    constexpr int kThreads = LANES > kBlock ? LANES : kBlock;
    constexpr int kRows = kThreads / LANES;
    constexpr int kCols = LANES * NV * V;
    // rows of several wavefronts: their exchange; others: the wavefronts' sums of the weight's gradient
    __shared__ float lds[LANES > kWave ? 4 * (LANES / kWave) : kWavesPerBlock * kCols];
    RowLanes<LANES> lanes(lds);
    const int lane = static_cast<int>(threadIdx.x) % LANES;
    const int64_t n = rows_of(a.num_rows, a.cap_rows);
    const int dim = a.dim;
    const bool full = dim == LANES * NV * V;               // every lane's vectors are its own
    float w[NV][V], gw[NV][V];
    Span<V> at[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        at[k] = Span<V>(k * LANES + lane, dim);
        load_weight(a.weight, at[k], dim, w[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) gw[k][j] = 0.f;
    }
    struct Row {
        W s[NV], g[NV], gs[NV];
    };
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        Row v;
        const T *sr = static_cast<const T *>(a.s) + row * a.s_stride;
        const T *gr = static_cast<const T *>(a.grad_y) + row * a.gy_stride;
        const T *gs = static_cast<const T *>(a.grad_sum) + row * a.gs_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            v.s[k] = load_span(sr, at[k], dim);
            v.g[k] = load_span(gr, at[k], dim);
            if (a.grad_sum) v.gs[k] = load_span(gs, at[k], dim);
        }
        return v;
    };
    // A row is on its way while the one before is worked on, if the registers hold both.
    constexpr bool kAhead = kThreads < 1024 || NV * V < 16;
    const int64_t step = int64_t(gridDim.x) * kRows;
    int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
    Row next;
    if (kAhead && row < n) next = load(row);
    for (; row < n; row += step) {
        Row v = kAhead ? next : load(row);
        if (kAhead && row + step < n) next = load(row + step);
        if (!full) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v.s[k][j] = at[k].mine(j) ? v.s[k][j] : static_cast<T>(0.f);
                    v.g[k][j] = at[k].mine(j) ? v.g[k][j] : static_cast<T>(0.f);
                }
        }
        if (!full) {                                       // (after a row's loads are on their way: before, they would wait for the weight's)
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (at[k].skip > 0)
#pragma unroll
                    for (int j = 0; j < V; ++j) w[k][j] = at[k].mine(j) ? w[k][j] : 0.f;
        }
        float squares = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float p = 0.f, d = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float s = static_cast<float>(v.s[k][j]);
                p += s * s;
                d += static_cast<float>(v.g[k][j]) * w[k][j] * s;
            }
            squares += p;
            dot += d;
        }
        lanes.sum_both(&squares, &dot);
        float mean = of_wave<LANES>(squares) / static_cast<float>(dim) + a.eps, unit = 1.f;
        dot = of_wave<LANES>(dot);
        if (ballot64(odd_mean(mean))) {
            unit = row_unit(mean);
            squares = dot = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float s = static_cast<float>(v.s[k][j]) * unit;
                    squares += s * s;
                    dot += static_cast<float>(v.g[k][j]) * w[k][j] * s;
                }
            lanes.sum_both(&squares, &dot);
            mean = unit_mean(of_wave<LANES>(squares), dim, a.eps, unit);
            dot = of_wave<LANES>(dot);
        }
        float r = 1.0f / sqrtf(mean);
        const float c = r * r * (dot / static_cast<float>(dim)) * unit;
        r *= unit;
        T *gx = static_cast<T *>(a.grad_x) + row * a.gx_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float out[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float s = static_cast<float>(v.s[k][j]), g = static_cast<float>(v.g[k][j]);
                gw[k][j] += g * (s * r);
                out[j] = r * (g * w[k][j] - c * s);
                if (a.grad_sum) out[j] += static_cast<float>(v.gs[k][j]);
            }
            store_span<PAST>(gx, at[k], dim, out);
        }
    }
    if (!a.parts) return;
    float *part = a.parts + int64_t(blockIdx.x) * dim;
    if constexpr (LANES > kWave) {                         // the workgroup is one row's: nothing to join
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int col = at[k].base + j;
                if (at[k].mine(j) && col < dim) part[col] = gw[k][j];
            }
    } else {
        const int wave = static_cast<int>(threadIdx.x) >> 6;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v = gw[k][j];
#pragma unroll
                for (int off = LANES; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
                if (lane_id() < LANES && at[k].mine(j)) lds[wave * kCols + at[k].base + j] = v;
            }
        __syncthreads();
        for (int col = static_cast<int>(threadIdx.x); col < dim; col += kThreads) {
            float v = lds[col];
#pragma unroll
            for (int k = 1; k < kWavesPerBlock; ++k) v += lds[k * kCols + col];
            part[col] = v;
        }
    }
}

template <typename T>
int launch_norm(mqg_ctx *ctx, const NormArgs &a, hipStream_t s) {
    const RowShape sh = row_shape(a.dim, Vec<T>::kLen, a.cap_rows);
    const int64_t cells = a.cap_rows * a.dim, arrays = 1 + (a.residual != nullptr) + (a.sum != nullptr) + (a.y != nullptr);
    const bool past = cells * (arrays * int64_t(sizeof(T)) + (a.q != nullptr)) >= kPastBytes;
    const int threads = std::max(sh.lanes, kBlock);
    // A workgroup takes one set of rows, of 16-bit rows, whose weight is twice as long as they are, several: 8,192 workgroups of 256 threads at most.
    // With at most 2,048, 8,192, 16,384 and no limit, us:  fp16 295,000 x 256 into e4m3 106, 101, 98, 100; 300,000 x 100 62, 57, 55, 55; 100,000 x 602 into rows and e4m3
    // 121, 110, 112, 121; bf16 1 M x 64 52, 42, 45, 55; 40,000 x 1,000 57, 55, 55, 56; 8,192^2 105, 105, 107, 108;  fp32 109,000 x 602 209, 193, 188, 189;
    // 20,000 x 2,048 120, 110, 105, 107; 295,000 x 256 into e4m3 221, 171, 170, 180; 300,000 x 100 113, 89, 90, 93 and without a residual 59, 48, 50, 65.
    const int64_t most = sizeof(T) == 4 ? (int64_t(1) << 31) - 1 : int64_t(8192) * kBlock / threads;
    const int64_t grid = std::min<int64_t>(std::min<int64_t>(ceil_div(a.cap_rows, threads / sh.lanes), most), ((int64_t(1) << 32) - 1) / threads);
#define MQG_GO(T, L, N)                                                                                                        \
    do {                                                                                                                       \
        if (past) MQG_LAUNCH(ctx, "k_rms_norm", s, (k_rms_norm<T, L, N, true><<<static_cast<uint32_t>(grid), threads, 0, s>>>(a)));  \
        else MQG_LAUNCH(ctx, "k_rms_norm", s, (k_rms_norm<T, L, N, false><<<static_cast<uint32_t>(grid), threads, 0, s>>>(a)));      \
    } while (0)
    MQG_NORM_SHAPES(T, MQG_GO)
#undef MQG_GO
    return MQG_OK;
}

template <typename T>
int launch_norm_backward(mqg_ctx *ctx, NormGradArgs a, float *grad_weight, hipStream_t s) {
    const RowShape sh = row_shape(a.dim, Vec<T>::kLen, a.cap_rows);
    const int threads = std::max(sh.lanes, kBlock);
    const int64_t sets = ceil_div(a.cap_rows, threads / sh.lanes);
    // Rows of a few rounds are one workgroup's, whose sum is the gradient, and the second launch falls away: 1 to 64 rows of 64 fp32 9.1 to 9.5 us a call
    // against 6.7 to 7.2, four of 1,024 bf16 9.2 against 6.6, two of 8,192 9.3 against 8.5.  Further rounds cost more than they save: eight rows of 1,024
    // 9.1 against 9.0 (waited for: 20.9 against 23.2), four of 8,192 9.3 against 11.7.
    const bool alone = grad_weight && sets > 0 && sets <= (sh.lanes <= kBlock ? 4 : 2);
    const int grid = alone ? 1 : static_cast<int>(std::min<int64_t>(sets, kNormParts));
    const bool past = a.cap_rows * a.dim * (a.grad_sum ? 4 : 3) * int64_t(sizeof(T)) >= kPastBytes;
    if (alone) {
        a.parts = grad_weight;
    } else if (grad_weight) {
        int rc = ensure_layer_scratch(ctx, norm_scratch_bytes(a.dim), s, "mqg_rms_norm_backward");
        if (rc != MQG_OK) return rc;
        a.parts = reinterpret_cast<float *>(ctx->layer_scratch.data);
    }
#define MQG_GO(T, L, N)                                                                                                        \
    do {                                                                                                                       \
        if (past) MQG_LAUNCH(ctx, "k_rms_norm_backward", s, (k_rms_norm_backward<T, L, N, true><<<grid, threads, 0, s>>>(a)));      \
        else MQG_LAUNCH(ctx, "k_rms_norm_backward", s, (k_rms_norm_backward<T, L, N, false><<<grid, threads, 0, s>>>(a)));          \
    } while (0)
    if (grid > 0) {
        MQG_NORM_SHAPES(T, MQG_GO)
    }
#undef MQG_GO
    if (grad_weight && !alone)
        MQG_LAUNCH(ctx, "k_sum_parts", s,
                   (k_sum_parts<<<static_cast<int>(ceil_div(a.dim, kSumCols)), kSumThreads, 0, s>>>(a.parts, grid, a.dim, grad_weight, a.dim, nullptr)));
    return MQG_OK;
}

}  // namespace

int run_rms_norm(mqg_ctx *ctx, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight,
                 float eps, const int64_t *num_rows, int64_t cap_rows, int32_t dim, int32_t dtype, void *sum, int64_t sum_stride, void *y,
                 int64_t y_stride, void *q, int64_t q_stride, int32_t q_type, int32_t group, float *scale, int64_t scale_stride, hipStream_t s) {
    if (cap_rows == 0) return MQG_OK;
    const NormArgs a{x, residual, weight, num_rows, sum, y, static_cast<uint8_t *>(q), scale, x_stride, residual_stride, sum_stride,
                     y_stride, q_stride, scale_stride, cap_rows, eps, dim, q_type, group};
    if (dtype == MQG_F16) return launch_norm<F16>(ctx, a, s);
    if (dtype == MQG_BF16) return launch_norm<BF16>(ctx, a, s);
    return launch_norm<float>(ctx, a, s);
}

int run_rms_norm_backward(mqg_ctx *ctx, const void *grad_y, int64_t gy_stride, const void *sum, int64_t sum_stride, const float *weight,
                          const void *grad_sum, int64_t gs_stride, float eps, const int64_t *num_rows, int64_t cap_rows, int32_t dim,
                          int32_t dtype, void *grad_x, int64_t gx_stride, float *grad_weight, hipStream_t s) {
    const NormGradArgs a{grad_y, sum, grad_sum, weight, num_rows, grad_x, nullptr, gy_stride, sum_stride, gs_stride, gx_stride, cap_rows, eps, dim};
    if (dtype == MQG_F16) return launch_norm_backward<F16>(ctx, a, grad_weight, s);
    if (dtype == MQG_BF16) return launch_norm_backward<BF16>(ctx, a, grad_weight, s);
    return launch_norm_backward<float>(ctx, a, grad_weight, s);
}

}  // namespace mqg
