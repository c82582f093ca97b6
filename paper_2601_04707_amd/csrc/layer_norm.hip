// Layer norm of the rows between two layers, with the residual's addition and an output in 8 bits, and its backward.
//
//   forward    s = x + r,  d = s - mean(s),  y = d R w + b with R = 1/sqrt(mean(d^2) + eps),  8 bits as of the root-mean-square norm
//   backward   with u = d R and h = gy w:  gx = R (h - mean(h) - u mean(h u)) + gs,  gw = sum over rows of gy u,  gb = sum over rows of gy
//
// Both are bound by memory: every input is read once and every output written once, a row stays in registers in between, laid out over lanes as the other
// norm's rows are.  The mean is taken first and the squares are those of the differences from it, so that rows whose mean is large against their
// spread keep it; what the mean was off by (the differences' own mean, which the same exchange gives) is taken out of both.  So a row has two exchanges between lanes.
// Measured on buffers in turn, of the 6.2 TB/s that an elementwise kernel reads and writes at: forward 295,000 x 256 fp16 into e4m3 86 us = 6.2, 109,000 x 602 fp32 175 = 6.0,
// 8,192 x 8,192 bf16 92 = 5.8; backward 295,000 x 256 fp16 102 us = 5.9, 109,000 x 602 fp32 176 = 6.0, 8,192 x 8,192 bf16 103 to 108 = 5.0 to 5.2.  Of a million e4m3 values 0.8 to 1.4 are the
// neighbour of the one that the formula has in 64 bits (1.5 to 2.7 in elementary fp32 operations), of int8 1.9 to 2.2 (2.5 to 3.3).
#include <algorithm>

#include "norm_rows.h"

namespace mqg {

namespace {

// A call that moves more than the chip's memory-side cache holds goes past the caches, with its loads, too (buffers that it doesn't hold from the call before: 295,000 x 256 fp16
// into e4m3 98 -> 85 us, 109,000 x 602 fp32 197 with all through the caches, 188 with the stores past them, 175; its backward 204, 195, 176; 1 M x 64 bf16 94 -> 87; 40,000 x 1,000 bf16
// 57 either way).  Smaller ones leave their output there for the next reader.
constexpr int64_t kLayerPastBytes = int64_t(256) << 20;

struct LayerArgs {
    const void *x, *residual;
    const float *weight, *bias;
    const int64_t *num_rows;
    void *sum, *y;
    uint8_t *q;
    float *scale;
    int64_t x_stride, residual_stride, sum_stride, y_stride, q_stride, scale_stride;
    int64_t cap_rows;
    float eps, per_dim;               // per_dim: 1 / dim, by which means are taken (a division takes ten operations, in each of a row's lanes)
    int32_t dim, q_type, group;       // group: columns per scale, 0 = the row
};

// Sums and maxima that the lanes of a row find together, MOST at a time.  Rows of several wavefronts exchange through LDS: two buffers in turn, so that one
// barrier per exchange is enough (who writes a buffer again has passed the barrier behind which all have read it).
template <int LANES, int MOST>
struct RowExchange {
    static constexpr int kWaves = LANES / kWave;
    static constexpr int kRoom = LANES > kWave ? 2 * MOST * kWaves : 1;
    float *lds;
    int turn = 0;
    __device__ __forceinline__ explicit RowExchange(float *l) : lds(l) {}
    template <int N>
    __device__ __forceinline__ void sums(float (&v)[N]) {
        static_assert(N <= MOST, "room for MOST values of every wavefront");
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i], LANES < kWave ? LANES : kWave);
        if constexpr (LANES > kWave) {
            float *buf = lds + turn * MOST * kWaves;
            turn ^= 1;
            if (lane_id() == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) buf[N * (threadIdx.x >> 6) + i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = buf[i];
#pragma unroll
            for (int k = 1; k < kWaves; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += buf[N * k + i];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = of_wave<LANES>(v[i]);
    }
    // the first lane's, in all of them
    __device__ __forceinline__ float first(float v) {
        if constexpr (LANES <= kWave) return of_wave<LANES>(__shfl(v, lane_id() & ~(LANES - 1), kWave));
        float *buf = lds + turn * MOST * kWaves;
        turn ^= 1;
        if (threadIdx.x == 0) buf[0] = v;
        __syncthreads();
        return buf[0];
    }
    __device__ __forceinline__ uint32_t max(uint32_t v) {
        v = lanes_max(v, LANES < kWave ? LANES : kWave);
        if constexpr (LANES > kWave) {
            float *buf = lds + turn * MOST * kWaves;
            turn ^= 1;
            if (lane_id() == 0) buf[threadIdx.x >> 6] = __uint_as_float(v);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kWaves; ++k) v = max_u32(v, __float_as_uint(buf[k]));
        }
        return v;
    }
};

// A lane's vectors of a row, and which of their elements are its own: bit j of own[k].
template <int LANES, int NV, int V>
struct RowPlaces {
    Span<V> at[NV];
    uint32_t own[NV];
    static constexpr uint32_t kAll = (1u << V) - 1;
    __device__ __forceinline__ RowPlaces(int lane, int dim) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            at[k] = Span<V>(k * LANES + lane, dim);
            own[k] = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) own[k] |= at[k].mine(j) && at[k].base + j < dim ? 1u << j : 0u;
        }
    }
    // f(j) for the elements of vector k that are its own
    template <typename F>
    __device__ __forceinline__ void for_own(int k, F f) const {
        if (own[k] == kAll) {
#pragma unroll
            for (int j = 0; j < V; ++j) f(j);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if ((own[k] >> j) & 1) f(j);
        }
    }
    // Others' elements become zero.
    __device__ __forceinline__ void keep_own(float (&v)[NV][V]) const {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (own[k] != kAll) {
#pragma unroll
                for (int j = 0; j < V; ++j) v[k][j] = (own[k] >> j) & 1 ? v[k][j] : 0.f;
            }
    }
};

// A thread's own sums, in registers, or, IN_LDS, in places of LDS that no other thread reads or writes: wide rows leave no registers for them.
template <int NV, int V, int THREADS, bool IN_LDS>
struct OwnSums {
    typedef float Quad __attribute__((ext_vector_type(4)));
    static constexpr int kQuads = IN_LDS ? NV * V / 4 * THREADS : 1;
    float v[IN_LDS ? 1 : NV][V];
    Quad *lds;
    __device__ __forceinline__ explicit OwnSums(Quad *l) : lds(l + threadIdx.x) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const float zeros[V] = {};
            put(k, zeros);
        }
    }
    __device__ __forceinline__ void get(int k, float (&out)[V]) const {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = IN_LDS ? lds[(k * V / 4 + j / 4) * THREADS][j % 4] : v[IN_LDS ? 0 : k][j];
    }
    __device__ __forceinline__ void put(int k, const float (&in)[V]) {
        if constexpr (IN_LDS) {
#pragma unroll
            for (int h = 0; h < V / 4; ++h) lds[(k * V / 4 + h) * THREADS] = Quad{in[4 * h], in[4 * h + 1], in[4 * h + 2], in[4 * h + 3]};
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[k][j] = in[j];
        }
    }
};

// The compiler forms nothing of the vectors beforehand and keeps it: a row waits as it was loaded.
template <typename W, int NV>
__device__ __forceinline__ void as_loaded(W (&v)[NV]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) asm volatile("" : "+v"(v[k]));
}

// How a group is taken to 8 bits: by max|y| / top as it is before it is rounded to the scale, in two terms, so that one rounding of those that can bring a value to the other side of a
// border falls away.  most and NaN as of the other norm.
struct FineScale {
    float scale, lo, inv;
};
__device__ __forceinline__ FineScale fine_scale(uint32_t most, float top) {
    const float m = __uint_as_float(most), per_top = 1.0f / top, t = m / top;
    if (!(t < __uint_as_float(0x7F800000u))) {
        const float nan = __uint_as_float(0x7FC00000u);
        return {nan, nan, nan};
    }
    if (!(t > 0x1p-100f)) {                                // (its second term would be below 32 bits' numbers)
        const float least = fmaxf(t, 0x1p-126f);
        return {least, 0.f, 1.0f / least};
    }
    return {t, fmaf(-t, top, m) * per_top, 1.0f / t};
}
template <int V>
__device__ __forceinline__ void to_8bit(const float (&z)[V], const FineScale &s, int q_type, uint32_t (&w)[V / 4]) {
    float y[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float quot = z[j] * s.inv;
        y[j] = fmaf(fmaf(-quot, s.lo, fmaf(-quot, s.scale, z[j])), s.inv, quot);
    }
    pack_8bit(y, s.scale == s.scale, q_type, w);
}

template <int V>
__device__ __forceinline__ void load_bias(const float *b, const Span<V> &at, int dim, float (&out)[V]) {
    if (b) {
        load_weight(b, at, dim, out);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = 0.f;
    }
}

// A mean, rounded: joined with the subtraction that follows it, it would be another one there than where it is used again.
__device__ __forceinline__ float mean_of(float sum, float per_dim) {
#pragma clang fp contract(off)
    return sum * per_dim;
}
// The variance of differences d from a mean that is off by their own mean c.  (A variance that is no number stays none.)
__device__ __forceinline__ float variance(float sum, float squares, float per_dim, float *c) {
    *c = mean_of(sum, per_dim);
    const float var = squares * per_dim - *c * *c;
    return var < 0.f ? 0.f : var;
}
// One over the root of 2^-100 to 2^100, to one unit of its last place: the card's, and the rest of its error.
__device__ __forceinline__ float reciprocal_root(float v) {
    const float y = __builtin_amdgcn_rsqf(v);
    return fmaf(y, 0.5f * fmaf(-v * y, y, 1.f), y);
}
// Rows that are taken again: the variance may have lost terms at either end of 32 bits' range, or the mean was off by as much as the row spreads (a row of
// equal values is off by its mean's rounding, and spreads not at all).  Then the differences are formed from the row's first value, exactly where they are small against it,
// times two powers of two: (s low - s0 low) high.  |s| up to 2^128 becomes up to 2^48, and variances of 2^100 and more 2^-60 and more; spreads of 2^-149 to 2^-50 become
// 2^-59 to 2^40.
struct Unit {
    float low, high;
};
// (c^2 and the variance of small values may both be below 32 bits' numbers, and read zero)
__device__ __forceinline__ bool odd_row(float var, float eps, float c) { return odd_mean(var + eps) || (c * c >= var && c != 0.f); }
// A mean that is off by c, far more than the row spreads, leaves nothing of the variance beside c^2: it may read zero where the row spreads up to 2^-8 c.  Such a row's values differ by
// 2^-13 c or more (a last place of s; c is 2^-11 of the mean at most), and so it is by c that it is known to be none of the smallest: its squares would leave 32 bits' range times 2^180.
__device__ __forceinline__ Unit odd_unit(float mean, float c) {
    return mean < 0x1p-100f && c * c < 0x1p-66f ? Unit{1.f, 0x1p+90f} : mean <= 0x1p+100f ? Unit{1.f, 1.f} : Unit{0x1p-80f, 1.f};
}
// The variance of the row times unit, and eps, or infinity, whose factor is 0, where the row's own factor is above 32 bits' numbers: rows of equal values without an
// epsilon, and such as spread less than 2^-128.
__device__ __forceinline__ float unit_variance(float var, float eps, float unit) {
    const float v = var + eps * unit * unit;
    return sqrtf(v) < unit * 0x1p-128f || v == 0.f ? __uint_as_float(0x7F800000u) : v;
}

template <typename T, int LANES, int NV, bool PAST>
__global__ void __launch_bounds__(LANES > kBlock ? LANES : kBlock)
k_layer_norm(LayerArgs a) {
    constexpr int V = Vec<T>::kLen;
    constexpr int kThreads = LANES > kBlock ? LANES : kBlock;
    constexpr int kRows = kThreads / LANES;                // rows of a workgroup
    using Exchange = RowExchange<LANES, 2>;
    __shared__ float lds[Exchange::kRoom];
    Exchange lanes(lds);
    const int lane = static_cast<int>(threadIdx.x) % LANES;
    const int64_t n = rows_of(a.num_rows, a.cap_rows);
    const int dim = a.dim;
    const float top = a.q_type == MQG_Q_E4M3 ? 448.f : 127.f;
    const int group_lanes = a.group / V;                   // lanes that share a scale, 0 = the row's
    const RowPlaces<LANES, NV, V> places(lane, dim);
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_weight(a.weight, places.at[k], dim, w[k]);
        load_bias(a.bias, places.at[k], dim, b[k]);
    }
    using W = typename Vec<T>::Whole;
    W raw[NV], more[NV];
    constexpr bool kAhead = kThreads < 1024 || NV * V < 16;    // a row is on its way while the one before is worked on, if the registers hold both
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *r0 = static_cast<const T *>(a.residual) + row * a.residual_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            raw[k] = load_span<PAST>(x, places.at[k], dim);
            if (a.residual) more[k] = load_span<PAST>(r0, places.at[k], dim);
        }
    };
    const int64_t step = int64_t(gridDim.x) * kRows;
    int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
    if (kAhead && row < n) load(row);
    for (; row < n; row += step) {
        if (!kAhead) load(row);
        float s[NV][V];
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[k][j] = static_cast<float>(raw[k][j]);
                if (a.residual) s[k][j] += static_cast<float>(more[k][j]);
            }
        if (kAhead && row + step < n) load(row + step);
        if (a.sum) {
            T *sum = static_cast<T *>(a.sum) + row * a.sum_stride;
#pragma unroll
            for (int k = 0; k < NV; ++k) store_span<PAST>(sum, places.at[k], dim, s[k]);
        }
        places.keep_own(s);
        float centre, var;                                 // the mean but for its error, which is taken out of the variance here and of the values below
        float c;
        auto stats = [&]() __attribute__((always_inline)) {
            float total[1] = {0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float part = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) part += s[k][j];
                total[0] += part;
            }
            lanes.sums(total);
            centre = mean_of(total[0], a.per_dim);
            // Of 16-bit rows a mean of 12 bits, from which the differences are exact; the rest of it is theirs, c.
            if (sizeof(T) == 2) centre = __uint_as_float(__float_as_uint(centre) & 0xFFFFF000u);
            float both[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float part = 0.f, squares = 0.f;
                places.for_own(k, [&](int j) __attribute__((always_inline)) {
                    const float d = s[k][j] - centre;
                    part += d;
                    squares += d * d;
                });
                both[0] += part;
                both[1] += squares;
            }
            lanes.sums(both);
            var = variance(both[0], both[1], a.per_dim, &c);
        };
        stats();
        float r;
        if (!odd_row(var, a.eps, c)) {                     // (the same in all lanes of a row)
            r = reciprocal_root(var + a.eps);
        } else {
            const Unit u = odd_unit(var + a.eps, c);
            const float s0 = lanes.first(s[0][0]) * u.low;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) s[k][j] = (s[k][j] * u.low - s0) * u.high;
            places.keep_own(s);
            stats();
            r = 1.0f / sqrtf(unit_variance(var, a.eps, u.low * u.high));
        }
        const float cr = c * r;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s[k][j] = fmaf(fmaf(s[k][j] - centre, r, -cr), w[k][j], b[k][j]);
        if (a.y) {
            T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
            for (int k = 0; k < NV; ++k) store_span<PAST>(y, places.at[k], dim, s[k]);
        }
        if (!a.q) continue;
        uint8_t *q = a.q + row * a.q_stride;
        float *scale = a.scale + row * a.scale_stride;
        places.keep_own(s);
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
            const FineScale sc = fine_scale(lanes.max(m), top);
            if (lane == 0) scale[0] = sc.scale;
#pragma unroll
            for (int k = 0; k < NV; ++k) store_q(q, places.at[k], dim, s[k], sc, a.q_type);
        } else {
            const int width = group_lanes < LANES ? group_lanes : LANES;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const FineScale sc = fine_scale(lanes_max(most[k], width), top);
                const int i = k * LANES + lane;
                if (lane % width == 0 && i * V < dim) scale[i / group_lanes] = sc.scale;
                store_q(q, places.at[k], dim, s[k], sc, a.q_type);
            }
        }
    }
}

struct LayerGradArgs {
    const void *grad_y, *s, *grad_sum;
    const float *weight;
    const int64_t *num_rows;
    void *grad_x;
    float *weight_parts, *bias_parts;      // every workgroup's share of the two gradients, `pitch` apart; null if not wanted
    uint32_t *done;                        // few columns and workgroups: those that have left their shares, of which the last adds them all; else null
    float *sum, *sum_bias;                 // ... to the gradients (`split` columns of the first)
    int32_t split;
    int64_t gy_stride, s_stride, gs_stride, gx_stride, pitch;
    int64_t cap_rows;
    float eps, per_dim;
    int32_t dim;
};

template <typename T, int LANES, int NV, bool PAST>
__global__ void __launch_bounds__(LANES > kBlock ? LANES : kBlock)
k_layer_norm_backward(LayerGradArgs a) {
    using W = typename Vec<T>::Whole;
    constexpr int V = Vec<T>::kLen;
    constexpr int kThreads = LANES > kBlock ? LANES : kBlock;
    constexpr int kRows = kThreads / LANES;
    constexpr int kCols = LANES * NV * V;
    using Exchange = RowExchange<LANES, 3>;
    // rows of several wavefronts: their exchange; others: the wavefronts' sums of the two gradients
    __shared__ float lds[LANES > kWave ? Exchange::kRoom : kWavesPerBlock * kCols];
    Exchange lanes(lds);
    const int lane = static_cast<int>(threadIdx.x) % LANES;
    const int64_t n = rows_of(a.num_rows, a.cap_rows);
    const int dim = a.dim;
    const RowPlaces<LANES, NV, V> places(lane, dim);
    float w[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) load_weight(a.weight, places.at[k], dim, w[k]);
    constexpr bool kInLds = kThreads >= 1024 && NV >= 2;   // (rows of 16,384, with all loads through the caches: 4,000 of bf16 243 -> 166 us, 2,000 of fp32 207 -> 155; in LDS rows of 8,192 bf16 116 -> 137.  With loads past them 136 and 125)
    using Own = OwnSums<NV, V, kThreads, kInLds>;
    __shared__ typename Own::Quad own[2 * Own::kQuads];
    Own gw(own), gb(own + Own::kQuads);
    struct Row {
        W s[NV], g[NV], gs[NV];
    };
    const int64_t step = int64_t(gridDim.x) * kRows;
    int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
    const T *sr = static_cast<const T *>(a.s) + row * a.s_stride;
    const T *gr = static_cast<const T *>(a.grad_y) + row * a.gy_stride;
    const T *gs = static_cast<const T *>(a.grad_sum) + row * a.gs_stride;
    T *gx = static_cast<T *>(a.grad_x) + row * a.gx_stride;
    auto load = [&]() __attribute__((always_inline)) {
        Row v;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            v.s[k] = load_span<PAST>(sr, places.at[k], dim);
            v.g[k] = load_span<PAST>(gr, places.at[k], dim);
            if (a.grad_sum) v.gs[k] = load_span<PAST>(gs, places.at[k], dim);
        }
        sr += step * a.s_stride;
        gr += step * a.gy_stride;
        gs += step * a.gs_stride;
        return v;
    };
    constexpr bool kOpaque = kInLds;
    // A row is on its way while the one before is worked on, if the registers hold both.
    constexpr bool kAhead = kThreads < 1024 || NV * V < 16;
    Row next;
    if (kAhead && row < n) next = load();
    for (; row < n; row += step) {
        Row v = kAhead ? next : load();
        if (kAhead && row + step < n) next = load();
        places.keep_own(w);                                // (here a row's loads are on their way: before, they would wait for the weight's)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (places.own[k] != places.kAll) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v.s[k][j] = (places.own[k] >> j) & 1 ? v.s[k][j] : static_cast<T>(0.f);
                    v.g[k][j] = (places.own[k] >> j) & 1 ? v.g[k][j] : static_cast<T>(0.f);
                }
            }
        float centre, c, var, h_mean, dot;                 // the mean but for its error c; the mean of h, and of h with the differences from the mean
        // Values are formed again where they are used: a row's registers hold it as it was loaded.  value(k, j): that of s
        auto stats = [&](auto value) __attribute__((always_inline)) {
            float before[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float p = 0.f, q = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    p += value(k, j);
                    q += static_cast<float>(v.g[k][j]) * w[k][j];
                }
                before[0] += p;
                before[1] += q;
            }
            lanes.sums(before);
            if (kOpaque) { as_loaded(v.s); as_loaded(v.g); }
            centre = mean_of(before[0], a.per_dim);
            h_mean = mean_of(before[1], a.per_dim);
            float then[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float p = 0.f, q = 0.f, t = 0.f;
                places.for_own(k, [&](int j) __attribute__((always_inline)) {
                    const float d = value(k, j) - centre;
                    p += d;
                    q += d * d;
                    t += static_cast<float>(v.g[k][j]) * w[k][j] * d;
                });
                then[0] += p;
                then[1] += q;
                then[2] += t;
            }
            lanes.sums(then);
            var = variance(then[0], then[1], a.per_dim, &c);
            if (kOpaque) { as_loaded(v.s); as_loaded(v.g); }
            dot = then[2] * a.per_dim - c * h_mean;
        };
        // r: that of the values that are taken; by: the row's own
        auto put_row = [&](auto value, float r, float by) __attribute__((always_inline)) {
            const float cr = c * r;
            dot *= r;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float out[V], sum_w[V], sum_b[V];
                gw.get(k, sum_w);
                gb.get(k, sum_b);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float u = fmaf(value(k, j) - centre, r, -cr), g = static_cast<float>(v.g[k][j]);
                    sum_w[j] = fmaf(g, u, sum_w[j]);
                    sum_b[j] += g;
                    out[j] = fmaf(-u, dot, g * w[k][j] - h_mean) * by;
                    if (a.grad_sum) out[j] += static_cast<float>(v.gs[k][j]);
                }
                gw.put(k, sum_w);
                gb.put(k, sum_b);
                store_span<PAST>(gx, places.at[k], dim, out);
            }
        };
        auto plain = [&](int k, int j) __attribute__((always_inline)) { return static_cast<float>(v.s[k][j]); };
        stats(plain);
        if (!odd_row(var, a.eps, c)) {
            const float r = reciprocal_root(var + a.eps);
            put_row(plain, r, r);
        } else {
            const Unit u = odd_unit(var + a.eps, c);
            const float s0 = lanes.first(plain(0, 0)) * u.low;
            auto scaled = [&](int k, int j) __attribute__((always_inline)) {
                const float d = (static_cast<float>(v.s[k][j]) * u.low - s0) * u.high;
                return (places.own[k] >> j) & 1 ? d : 0.f;
            };
            stats(scaled);
            const float unit = u.low * u.high, r = 1.0f / sqrtf(unit_variance(var, a.eps, unit));
            // (of equal values so large that their sums leave 32 bits' range: their differences are zeros, whatever r is, but eps is below 32 bits' numbers times unit^2)
            put_row(scaled, r, unit < 1.f && var == 0.f && a.eps > 0.f ? 1.0f / sqrtf(a.eps) : r * unit);
        }
        gx += step * a.gx_stride;
    }
    // The workgroup's share of a gradient.
    auto put = [&](float *parts, const Own &sums) __attribute__((always_inline)) {
        if (!parts) return;
        float v[NV][V];
#pragma unroll
        for (int k = 0; k < NV; ++k) sums.get(k, v[k]);
        float *part = parts + int64_t(blockIdx.x) * a.pitch;
        if constexpr (LANES > kWave) {                     // the workgroup is one row's: nothing to join
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if ((places.own[k] >> j) & 1) part[places.at[k].base + j] = v[k][j];
        } else {
            const int wave = static_cast<int>(threadIdx.x) >> 6;
            __syncthreads();                               // the other gradient's sums are read
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float x = v[k][j];
#pragma unroll
                    for (int off = LANES; off < kWave; off <<= 1) x += __shfl_xor(x, off, kWave);
                    if (lane_id() < LANES && ((places.own[k] >> j) & 1)) lds[wave * kCols + places.at[k].base + j] = x;
                }
            __syncthreads();
            for (int col = static_cast<int>(threadIdx.x); col < dim; col += kThreads) {
                float x = lds[col];
#pragma unroll
                for (int k = 1; k < kWavesPerBlock; ++k) x += lds[k * kCols + col];
                part[col] = x;
            }
        }
    };
    put(a.weight_parts, gw);
    put(a.bias_parts, gb);
    if constexpr (LANES <= kWave) {
        if (!a.done) return;
        __shared__ bool last;
        __shared__ float joined[kThreads];
        const int tid = static_cast<int>(threadIdx.x), cols = static_cast<int>(a.pitch), num = static_cast<int>(gridDim.x);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent"); // (every wavefront's share, past its die's L2)
        __syncthreads();
        if (tid == 0) last = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
        __syncthreads();
        if (!last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        if (tid == 0) __hip_atomic_store(a.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // as many threads to a column as there are, each of which takes shares in turn; their sums in order
        const float *parts = a.weight_parts ? a.weight_parts : a.bias_parts;
        const int turns = kThreads / (2 * a.split), turn = tid / cols, col = tid % cols;     // (the same whether one gradient is wanted or both)
        constexpr int kOnTheWay = 16;
        float x = 0.f;
        for (int p0 = turn; turn < turns && p0 < num; p0 += kOnTheWay * turns) {
            float y[kOnTheWay];
#pragma unroll
            for (int k = 0; k < kOnTheWay; ++k) y[k] = p0 + k * turns < num ? parts[(p0 + k * turns) * cols + col] : 0.f;
#pragma unroll
            for (int k = 0; k < kOnTheWay; ++k) x += y[k];
        }
        joined[tid] = x;
        __syncthreads();
        if (tid >= cols) return;
        for (int k = 1; k < turns; ++k) x += joined[k * cols + tid];
        *(tid < a.split ? a.sum + tid : a.sum_bias + (tid - a.split)) = x;
    }
}

template <typename T>
int launch_layer_norm(mqg_ctx *ctx, const LayerArgs &a, hipStream_t s) {
    const RowShape sh = row_shape(a.dim, Vec<T>::kLen, a.cap_rows);
    const int64_t cells = a.cap_rows * a.dim, arrays = 1 + (a.residual != nullptr) + (a.sum != nullptr) + (a.y != nullptr);
    const bool past = cells * (arrays * int64_t(sizeof(T)) + (a.q != nullptr)) >= kLayerPastBytes;
    const int threads = std::max(sh.lanes, kBlock);
    // Several sets of rows to a workgroup, which reads weight and bias once: 109,000 x 602 fp32 with 2,048, 4,096, 16,384 workgroups of 256 threads 207, 204 and 190 us,
    // without a limit 201; 300,000 x 100 101, 95, 87 and 97; 295,000 x 256 fp16 into e4m3 with 2,048, 4,096 and 8,192 111, 108 and 101.  The longest fp32 rows, of which no second
    // one is on its way, 4,000 x 16,384: 186 with 1,024 of 1,024 threads, 214 with one a row.
    const bool longest = threads == 1024 && sh.nv > 2;
    const int64_t most = int64_t(sizeof(T) == 4 && !longest ? 16384 : longest ? 4096 : 8192) * kBlock / threads;
    const int64_t grid = std::min<int64_t>(std::min<int64_t>(ceil_div(a.cap_rows, threads / sh.lanes), most), ((int64_t(1) << 32) - 1) / threads);
#define MQG_GO(T, L, N)                                                                                                            \
    do {                                                                                                                           \
        if (past) MQG_LAUNCH(ctx, "k_layer_norm", s, (k_layer_norm<T, L, N, true><<<static_cast<uint32_t>(grid), threads, 0, s>>>(a)));  \
        else MQG_LAUNCH(ctx, "k_layer_norm", s, (k_layer_norm<T, L, N, false><<<static_cast<uint32_t>(grid), threads, 0, s>>>(a)));      \
    } while (0)
    MQG_NORM_SHAPES(T, MQG_GO)
#undef MQG_GO
    return MQG_OK;
}

// How a backward's rows are laid out: those of 16 bits that would take three or four vectors of a wavefront's lanes have four wavefronts (registers for one row on its way
// beside the sums: 20,000 x 2,000 bf16 90 -> 72 us; 30,000 x 1,500 90 -> 86).
RowShape grad_shape(int dim, int vec, int64_t rows) {
    const RowShape sh = row_shape(dim, vec, rows);
    return sh.lanes == kWave && sh.nv * vec > 16 ? RowShape{256, 1} : sh;
}
// Workgroups of a backward at most, each of which leaves its share of the gradients: as many as are on the chip together for the longest rows (8,192 x 8,192
// bf16: 256 103 us, 512 116) and for those of a wavefront (109,000 x 602 fp32: 512 176, 768 203), more for shorter ones, whose waits want others to fill them (258,000 x 174 bf16 512 107, 768
// 87, 1,024 80; 500,000 x 64 fp32 768 87, 1,024 91; 295,000 x 256 fp16 512 98, 768 102, 1,024 110; 2 M x 16 bf16 512 79, 768 73, 1,024 66), and for those of four
// wavefronts (20,000 x 2,000: 512 80, 1,024 73).
int grad_parts(const RowShape &sh) {
    if (sh.lanes <= 8 || sh.lanes == 256) return 1024;
    if (sh.lanes <= 32) return 768;
    return sh.lanes * sh.nv >= 1024 ? 256 : 512;
}

}  // namespace

// The shares of both gradients of rows of up to dim columns, of any type and number: a layout's widest rows have the most (few rows have a workgroup each at most).
int64_t layer_norm_scratch_bytes(int32_t dim) {
    int64_t floats = 2 * int64_t(kFewRows) * dim;
    for (int vec : {4, 8})
        for (int vecs : {4, 8, 16, 32, 64, 128, 192, 256, 512, 1024, 2048, 4096}) {
            const int widest = std::min(vecs * vec, dim);
            floats = std::max(floats, 2 * int64_t(widest) * grad_parts(grad_shape(widest, vec, INT64_MAX)));
            if (widest == dim) break;
        }
    return floats * int64_t(sizeof(float));
}

namespace {

constexpr int kJoinGrid = 32;         // workgroups whose shares the last of them adds

#define MQG_GRAD_SHAPES(T, GO)                                     \
    switch (sh.lanes) {                                            \
        case 4: GO(T, 4, 1); break;                                \
        case 8: GO(T, 8, 1); break;                                \
        case 16: GO(T, 16, 1); break;                              \
        case 32: GO(T, 32, 1); break;                              \
        case 64:                                                   \
            if (sh.nv == 1) GO(T, 64, 1);                          \
            else if (sh.nv == 2) GO(T, 64, 2);                     \
            else if constexpr (sizeof(T) == 4) {                   \
                if (sh.nv == 3) GO(T, 64, 3);                      \
                else GO(T, 64, 4);                                 \
            }                                                      \
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

template <typename T>
int launch_layer_norm_backward(mqg_ctx *ctx, LayerGradArgs a, float *grad_weight, float *grad_bias, hipStream_t s) {
    const RowShape sh = grad_shape(a.dim, Vec<T>::kLen, a.cap_rows);
    const int threads = std::max(sh.lanes, kBlock);
    const int64_t sets = ceil_div(a.cap_rows, threads / sh.lanes);
    const int wanted = (grad_weight != nullptr) + (grad_bias != nullptr);
    // Rows of a few rounds are one workgroup's, whose sums are the gradients, and the second launch falls away.
    const bool alone = wanted && sets > 0 && sets <= (sh.lanes <= kBlock ? 4 : 2);
    const int grid = alone ? 1 : static_cast<int>(std::min<int64_t>(sets, grad_parts(sh)));
    const bool past = a.cap_rows * a.dim * (a.grad_sum ? 4 : 3) * int64_t(sizeof(T)) >= kLayerPastBytes;
    a.pitch = int64_t(wanted) * a.dim;
    float *parts = nullptr;
    if (alone) {
        a.weight_parts = grad_weight;
        a.bias_parts = grad_bias;
    } else if (wanted) {
        int rc = ensure_layer_scratch(ctx, std::max(layer_norm_scratch_bytes(a.dim), grid * a.pitch * int64_t(sizeof(float))), s, "mqg_layer_norm_backward");
        if (rc != MQG_OK) return rc;
        parts = reinterpret_cast<float *>(ctx->layer_scratch.data);
        a.weight_parts = grad_weight ? parts : nullptr;
        a.bias_parts = grad_bias ? parts + (grad_weight ? a.dim : 0) : nullptr;
    }
    // The join of few shares of few columns in the last workgroup saves a launch, but every workgroup waits until its share is past its die: 300 x 64 bf16, 19 workgroups, 7.7 us a call
    // against 10.9, 1,400 x 64 fp32, 88, 10.8 either way, 1,000 x 128, 125, 16.1 against 10.9.
    const int cols = wanted * a.dim;
    const bool join = parts && grid > 0 && grid <= kJoinGrid && 2 * a.dim <= kBlock && threads == kBlock;
    if (join) {
        a.done = reinterpret_cast<uint32_t *>(ctx->norm_parts + kGradNormParts) + 1;
        a.sum = grad_weight ? grad_weight : grad_bias;
        a.sum_bias = grad_bias;
        a.split = a.dim;
    }
#define MQG_GO(T, L, N)                                                                                                                  \
    do {                                                                                                                                 \
        if (past) MQG_LAUNCH(ctx, "k_layer_norm_backward", s, (k_layer_norm_backward<T, L, N, true><<<grid, threads, 0, s>>>(a)));            \
        else MQG_LAUNCH(ctx, "k_layer_norm_backward", s, (k_layer_norm_backward<T, L, N, false><<<grid, threads, 0, s>>>(a)));                \
    } while (0)
    if (grid > 0) {
        MQG_GRAD_SHAPES(T, MQG_GO)
    }
#undef MQG_GO
    if (parts && !join) {
        MQG_LAUNCH(ctx, "k_sum_parts", s,
                   (k_sum_parts<<<static_cast<int>(ceil_div(cols, kSumCols)), kSumThreads, 0, s>>>(parts, grid, cols, grad_weight ? grad_weight : grad_bias,
                                                                                                    a.dim, grad_bias)));
    }
    return MQG_OK;
}

}  // namespace

int run_layer_norm(mqg_ctx *ctx, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight, const float *bias,
                   float eps, const int64_t *num_rows, int64_t cap_rows, int32_t dim, int32_t dtype, void *sum, int64_t sum_stride, void *y,
                   int64_t y_stride, void *q, int64_t q_stride, int32_t q_type, int32_t group, float *scale, int64_t scale_stride, hipStream_t s) {
    if (cap_rows == 0) return MQG_OK;
    const LayerArgs a{x, residual, weight, bias, num_rows, sum, y, static_cast<uint8_t *>(q), scale, x_stride, residual_stride, sum_stride,
                      y_stride, q_stride, scale_stride, cap_rows, eps, 1.0f / static_cast<float>(dim), dim, q_type, group};
    if (dtype == MQG_F16) return launch_layer_norm<F16>(ctx, a, s);
    if (dtype == MQG_BF16) return launch_layer_norm<BF16>(ctx, a, s);
    return launch_layer_norm<float>(ctx, a, s);
}

int run_layer_norm_backward(mqg_ctx *ctx, const void *grad_y, int64_t gy_stride, const void *sum, int64_t sum_stride, const float *weight,
                            const void *grad_sum, int64_t gs_stride, float eps, const int64_t *num_rows, int64_t cap_rows, int32_t dim,
                            int32_t dtype, void *grad_x, int64_t gx_stride, float *grad_weight, float *grad_bias, hipStream_t s) {
    const LayerGradArgs a{grad_y, sum, grad_sum, weight, num_rows, grad_x, nullptr, nullptr, nullptr, nullptr, nullptr, 0, gy_stride, sum_stride, gs_stride, gx_stride, 0, cap_rows,
                          eps, 1.0f / static_cast<float>(dim), dim};
    if (dtype == MQG_F16) return launch_layer_norm_backward<F16>(ctx, a, grad_weight, grad_bias, s);
    if (dtype == MQG_BF16) return launch_layer_norm_backward<BF16>(ctx, a, grad_weight, grad_bias, s);
    return launch_layer_norm_backward<float>(ctx, a, grad_weight, grad_bias, s);
}

}  // namespace mqg
