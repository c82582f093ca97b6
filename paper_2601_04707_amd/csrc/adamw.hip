// The norm of all gradients, and the AdamW step of many tensors in a launch, with moments in 32 bits or in 8.
//
//   norm   n = mul sqrt(sum over all g^2),  scale = mul min(1, most / n)
//   step   g' = scale g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
//          w = (1 - lr decay) w - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
//   8 bits m and sqrt(v) of 128 elements in order as e4m3 values times a scale that is the block's own: the largest of each keeps 32 bits.  The root instead of
//          v itself: e4m3 reaches down to 2^-18 of its largest value, which is 2^-36 of v.  A root above zero that would round to zero becomes the least
//          value above it, so that no moment is divided by epsilon alone.
//
// Both are bound by memory: what is read is read once, what is written is written once.  The tensors' addresses and sizes come with the launch, 74 to 120 tensors at a
// time (and eight pairs of lr_scale and decay_scale: a list in which every few tensors have rates of their own takes more launches), so that nothing is copied to the device beforehand; a workgroup finds its tensor by a
// comparison in every lane.  Measured on buffers in turn, of the 6.2 TB/s
// that an elementwise kernel reads and writes at: 101 M elements with bf16 gradients and bf16 copies, moments in 32 bits 460 to 490 us = 5.8 to 6.15, in 8 bits 260 = 6.3 (of bf16
// weights without copies 167 = 6.1), packed one right after the other with odd sizes 470 and 308; the norm of 202 MB of bf16 36 = 5.6.  With
// the step's number read on the device (the millionth) every wavefront forms the two powers before its first load: 32 bits 447, 8 bits 398, of bf16 weights 239.
#include <algorithm>
#include <cmath>
#include <vector>

#include "common.h"
#include "layer_types.h"

namespace mqg {
namespace {

// Steps that move more than half of what the chip's memory-side cache holds go past the caches, with their loads, too: what lies between two steps of a program leaves nothing
// there (on buffers in turn: 12.8 M elements in 32 bits, 358 MB, 81 -> 69 us; with 8-bit moments and bf16 copies, 206 MB, 50 -> 46; 100 M, 2.8 GB, 517 -> 463.  3.2 M, 91 MB,
// 16.2 -> 19.3).  The norm's reads do where the gradients don't fit: the step reads those again (202 MB of them: norm and step 474, past the caches 504).
constexpr int64_t kStepPastBytes = int64_t(128) << 20, kNormPastBytes = int64_t(256) << 20;
constexpr int64_t kMostElems = int64_t(1) << 31;       // of a launch; longer tensors go in parts

// x + y of two products, each rounded by itself: 8-bit moments go from step to step, where one that falls to the other side of a rounding border is a sixteenth
// off, and so they are those of a program in elementary operations, whichever of them the compiler would join.
__device__ __forceinline__ float apart_add(float x, float y) {
#pragma clang fp contract(off)
    return x + y;
}

// Which of `count` tensors workgroup `group` belongs to: the last that begins at it or before.  MOST: how many there can be.
template <int MOST>
__device__ __forceinline__ int tensor_of(const uint32_t *first, int count, uint32_t group) {
    int before = 0;
#pragma unroll
    for (int k = 0; k < MOST; k += kWave) {
        const int i = k + lane_id();
        before += popc64(ballot64(i < count && first[i] <= group));
    }
    return __builtin_amdgcn_readfirstlane(before - 1);
}

// beta^t for t >= 1, by squaring
__host__ __device__ __forceinline__ double power(double beta, int64_t t) {
    double all = 1.0;
    for (double p = beta; t > 0; t >>= 1, p *= p)
        if (t & 1) all *= p;
    return all;
}

// How many elements before a tensor its first workgroup begins, so that each begins at a whole cache line of it.
constexpr int kLine = 128;
template <typename T>
int line_shift(const T *p) {
    return static_cast<int>(reinterpret_cast<uintptr_t>(p) % kLine / sizeof(T));
}

// What a launch of the step knows, 4 KB at most: a tensor's addresses (weight, gradient, m, v, then the copy and the scales if there are any),
// its first workgroup, the elements of its last one, and which of a few pairs of factors it has.
constexpr int kArgBytes = 4096, kFactors = 8;          // (a ninth pair begins another launch)
struct StepFactors {
    float size, keep;                    // lr / (1 - beta1^t), 1 - lr decay
    float lr_scale, decay_scale;
};
struct StepPlan {
    double lr, decay, beta1, beta2;
    int64_t host_step;
    const int64_t *step;                 // t and lr where the host does not know them
    const float *lr_dev, *grad_scale;
    float beta1_f, beta2_f, new1, new2;  // new: 1 - beta
    float root_by, eps;                  // 1 / sqrt(1 - beta2^t)
    int32_t count, copy_type;
    uint32_t groups;                     // workgroups of all tensors
    StepFactors factors[kFactors];
};
// The same on the host and on the device.
__host__ __device__ __forceinline__ float debiased_root_by(double beta2, int64_t t) { return 1.0f / sqrtf(static_cast<float>(1.0 - power(beta2, t))); }
__host__ __device__ __forceinline__ void set_factors(StepFactors &f, double lr, double decay, double beta1, int64_t t) {
    const double rate = lr * f.lr_scale;
    f.size = static_cast<float>(rate) / static_cast<float>(1.0 - power(beta1, t));
    f.keep = static_cast<float>(fma(-rate, decay * f.decay_scale, 1.0));
}
enum { kWeight, kGrad, kM, kV };
template <bool EIGHT, bool COPY>
struct StepArgs {
    static constexpr int kCopy = 4, kMScale = 4 + COPY, kVScale = 5 + COPY, kPointers = 4 + COPY + 2 * EIGHT;
    static constexpr int kHigh = (kPointers + 1) / 2;
    static constexpr int kTensors = (kArgBytes - static_cast<int>(sizeof(StepPlan))) / (4 * (kPointers + kHigh + 2));
    // (whole words, which are read by scalar loads)
    StepPlan plan;
    uint32_t low[kPointers][kTensors];   // addresses, of 48 bits; two of the high halves to a word
    uint32_t high[kHigh][kTensors];
    uint32_t first[kTensors];
    uint32_t rest[kTensors];             // the last workgroup's elements less one, factors << 16, shift << 24 (of moments in 32 bits: blocks of 8-bit ones are counted from the tensor's beginning)
    void set(int which, int tensor, const void *p) {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        const uint32_t half = static_cast<uint32_t>(at >> 32 & 0xFFFF);
        low[which][tensor] = static_cast<uint32_t>(at);
        high[which / 2][tensor] = which % 2 == 0 ? half : high[which / 2][tensor] | half << 16;       // (in order)
    }
    __device__ __forceinline__ void *get(int which, int tensor) const {
        const uint64_t at = static_cast<uint64_t>(high[which / 2][tensor] >> which % 2 * 16 & 0xFFFF) << 32 | low[which][tensor];
        return (void *)reinterpret_cast<__attribute__((address_space(1))) void *>(at);      // (global memory's: the general kind of load waits for LDS, too)
    }
};
static_assert(sizeof(StepArgs<true, true>) <= kArgBytes && sizeof(StepArgs<true, false>) <= kArgBytes && sizeof(StepArgs<false, true>) <= kArgBytes &&
              sizeof(StepArgs<false, false>) <= kArgBytes, "a launch's arguments");

template <typename T, int N>
struct Some {
    typedef T Whole __attribute__((ext_vector_type(N)));
    typedef Whole Any __attribute__((aligned(sizeof(T))));
};
// N elements of a tensor from i on, which may be below zero; zeros outside.  FULL: they are all there; PAST: not to be kept in the caches, here and below
template <bool PAST, bool FULL, int N, typename T>
__device__ __forceinline__ typename Some<T, N>::Whole load_some(const T *p, int64_t i, int64_t end) {
    typename Some<T, N>::Whole v;
    if (FULL || (i >= 0 && i + N <= end)) {
        if constexpr (PAST) v = __builtin_nontemporal_load(reinterpret_cast<const typename Some<T, N>::Any *>(p + i));
        else v = *reinterpret_cast<const typename Some<T, N>::Any *>(p + i);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = i + j >= 0 && i + j < end ? p[i + j] : static_cast<T>(0.f);
    }
    return v;
}
template <bool PAST, bool FULL, typename T, int N>
__device__ __forceinline__ void store_some(T *p, int64_t i, int64_t end, const float (&in)[N]) {
    typename Some<T, N>::Whole v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = static_cast<T>(in[j]);
    if (FULL || (i >= 0 && i + N <= end)) {
        if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<typename Some<T, N>::Any *>(p + i));
        else *reinterpret_cast<typename Some<T, N>::Any *>(p + i) = v;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i + j >= 0 && i + j < end) p[i + j] = v[j];
    }
}

// E e4m3 values, four to a word
template <int W>
struct Words {
    typedef uint32_t Whole __attribute__((ext_vector_type(W)));
    typedef Whole Any __attribute__((aligned(1)));
};
template <bool PAST, bool FULL, int E>
__device__ __forceinline__ typename Words<E / 4>::Whole load_8bit(const uint8_t *p, int64_t i, int64_t end) {
    typename Words<E / 4>::Whole w = 0;
    if (FULL || i + E <= end) {
        if constexpr (PAST) w = __builtin_nontemporal_load(reinterpret_cast<const typename Words<E / 4>::Any *>(p + i));
        else w = *reinterpret_cast<const typename Words<E / 4>::Any *>(p + i);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (i + j < end) w[j / 4] |= static_cast<uint32_t>(p[i + j]) << (8 * (j % 4));
    }
    return w;
}
template <int W, int E>
__device__ __forceinline__ void of_e4m3(uint32_t __attribute__((ext_vector_type(W))) w, float (&out)[E]) {
    static_assert(E == 4 * W, "four to a word");
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const int word = static_cast<int>(w[k]);
        out[4 * k] = __builtin_amdgcn_cvt_f32_fp8(word, 0);
        out[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8(word, 1);
        out[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8(word, 2);
        out[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8(word, 3);
    }
}
template <bool PAST, bool FULL, int E>
__device__ __forceinline__ void store_8bit(uint8_t *p, int64_t i, int64_t end, const float (&y)[E]) {
    typename Words<E / 4>::Whole w;
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
        const int half = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false);
        w[k] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2], y[4 * k + 3], half, true));
    }
    if (FULL || i + E <= end) {
        if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<typename Words<E / 4>::Any *>(p + i));
        else *reinterpret_cast<typename Words<E / 4>::Any *>(p + i) = w;
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (i + j < end) p[i + j] = static_cast<uint8_t>(w[j / 4] >> (8 * (j % 4)));
    }
}

// The square root, rounded to nearest: from the card's reciprocal root (one unit of its last place) by the remainder, for zero and 2^-100 to 2^126.
__device__ __forceinline__ float root_of(float v) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(v, 0x1p-100f)), root = v * y;
    return fmaf(fmaf(-root, root, v), 0.5f * y, root);
}
// An 8-bit block's scale, max / 448, and the division by it; scale NaN where the largest is not finite.
struct BlockScale {
    float scale, inv;
    __device__ __forceinline__ explicit BlockScale(float most) {
        const float s = fmaxf(most * (1.0f / 448.0f), 0x1p-126f);
        scale = most < __uint_as_float(0x7F800000u) ? s : __uint_as_float(0x7FC00000u);
        inv = 1.0f / scale;
    }
    // the quotient by the reciprocal, and its remainder's
    __device__ __forceinline__ float of(float x) const {
        const float q = x * inv;
        return fmaf(fmaf(-q, scale, x), inv, q);
    }
};
constexpr int kStepThreads = 128;
// A thread's elements.  Four 32-bit weights, or eight of 16 bits, are 16 bytes, and a wavefront's accesses to them a whole kilobyte.  101 M elements with bf16 gradients and copies: moments in
// 32 bits by fours 462 us, by eights 543, twice four 497; 8-bit ones by fours 259, twice four 270, by eights 309, with 64 and 256 threads 263 and 266; bf16 weights with 8-bit moments by
// eights 167, by fours 192.
template <typename TW, bool EIGHT>
struct StepShape {
    static constexpr int kElems = EIGHT ? 16 / static_cast<int>(sizeof(TW)) : 4;
    static constexpr int kGroup = kStepThreads * kElems;
    static constexpr int kScaleLanes = MQG_ADAMW_BLOCK / kElems;      // that share a scale
    static_assert(kGroup % MQG_ADAMW_BLOCK == 0 && kScaleLanes <= kWave, "a workgroup has whole blocks, a wavefront their lanes");
};

// What a workgroup's elements are stepped with
struct StepNumbers {
    float by, size, keep, beta1, beta2, new1, new2, root_by, eps;
    int32_t copy_type;
};
// One workgroup's elements of a tensor.  FULL: all of them are there; a bound at every access would have each load waited for before the next one.  LINES: the 8-bit moments
// begin at whole cache lines; where they don't, lines that two wavefronts share are read through the caches, once (twice four elements a thread: 101 M elements of odd tensors, one right after the
// other, 323 us and 355 past them; where they do, 277 and 269).
template <typename TW, typename TG, bool EIGHT, bool COPY, bool PAST, bool FULL, bool LINES>
__device__ __forceinline__ void step_group(const StepNumbers &n, void *const (&of)[StepArgs<EIGHT, COPY>::kPointers], int64_t i, int64_t end) {
    using Args = StepArgs<EIGHT, COPY>;
    using Shape = StepShape<TW, EIGHT>;
    constexpr int E = Shape::kElems;
    TW *weight = static_cast<TW *>(of[kWeight]);
    const TG *grad = static_cast<const TG *>(of[kGrad]);
    typename Some<TW, E>::Whole w_raw;
    typename Some<TG, E>::Whole g_raw;
    typename Some<float, E>::Whole m_raw, v_raw;
    typename Words<E / 4>::Whole m8, v8;
    float ms, vs;
    g_raw = load_some<PAST, FULL, E>(grad, i, end);
    if constexpr (EIGHT) {
        m8 = load_8bit<PAST && LINES, FULL, E>(static_cast<const uint8_t *>(of[kM]), i, end);
        v8 = load_8bit<PAST && LINES, FULL, E>(static_cast<const uint8_t *>(of[kV]), i, end);
        ms = FULL || i < end ? static_cast<const float *>(of[Args::kMScale])[i / MQG_ADAMW_BLOCK] : 0.f;
        vs = FULL || i < end ? static_cast<const float *>(of[Args::kVScale])[i / MQG_ADAMW_BLOCK] : 0.f;
    } else {
        m_raw = load_some<PAST, FULL, E>(static_cast<const float *>(of[kM]), i, end);
        v_raw = load_some<PAST, FULL, E>(static_cast<const float *>(of[kV]), i, end);
    }
    w_raw = load_some<PAST, FULL, E>(weight, i, end);
    float w[E], m[E], v[E], root[E];
    uint32_t most_m = 0, most_v = 0, least_v = ~0u;
    if constexpr (EIGHT) {
        of_e4m3<E / 4>(m8, m);
        of_e4m3<E / 4>(v8, v);
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        if constexpr (EIGHT) {
            m[j] *= ms;
            v[j] *= vs;
            v[j] *= v[j];
        } else {
            m[j] = m_raw[j];
            v[j] = v_raw[j];
        }
        const float g = static_cast<float>(g_raw[j]) * n.by;
        m[j] = apart_add(n.beta1 * m[j], n.new1 * g);
        v[j] = apart_add(n.beta2 * v[j], n.new2 * g * g);
        root[j] = root_of(v[j]);
        most_m = max_u32(most_m, __float_as_uint(m[j]) & 0x7FFFFFFFu);
        most_v = max_u32(most_v, __float_as_uint(v[j]));
        least_v = min(least_v, __float_as_uint(v[j]) - 1);         // (zero is none)
    }
    if (ballot64(least_v < __float_as_uint(0x1p-100f) - 1 || most_v > __float_as_uint(0x1p+126f))) {
#pragma unroll
        for (int j = 0; j < E; ++j) root[j] = sqrtf(v[j]);
    }
    const float none = n.eps == 0.f ? 0.f : -1.f;                  // the divisor that changes nothing
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const float under = fmaf(root[j], n.root_by, n.eps);
        // to one unit of its last place; no divisor but zero is below fp32's normal numbers
        const float inv = under == none ? 0.f : __builtin_amdgcn_rcpf(under);
        w[j] = fmaf(static_cast<float>(w_raw[j]), n.keep, -(n.size * m[j] * inv));
    }
    store_some<PAST, FULL>(weight, i, end, w);
    if constexpr (COPY) {
        void *copy = of[Args::kCopy];
        if (n.copy_type == MQG_F16) store_some<PAST, FULL>(static_cast<F16 *>(copy), i, end, w);
        else if (n.copy_type == MQG_BF16) store_some<PAST, FULL>(static_cast<BF16 *>(copy), i, end, w);
        else store_some<PAST, FULL>(static_cast<float *>(copy), i, end, w);
    }
    if constexpr (EIGHT) {
        const BlockScale sm(__uint_as_float(lanes_max(most_m, Shape::kScaleLanes)));
        const BlockScale sv(sqrtf(__uint_as_float(lanes_max(most_v, Shape::kScaleLanes))));
        if (threadIdx.x % Shape::kScaleLanes == 0 && (FULL || i < end)) {
            static_cast<float *>(of[Args::kMScale])[i / MQG_ADAMW_BLOCK] = sm.scale;
            static_cast<float *>(of[Args::kVScale])[i / MQG_ADAMW_BLOCK] = sv.scale;
        }
        float y[E];
#pragma unroll
        for (int j = 0; j < E; ++j) y[j] = sm.of(m[j]);
        store_8bit<PAST, FULL>(static_cast<uint8_t *>(of[kM]), i, end, y);
#pragma unroll
        for (int j = 0; j < E; ++j) y[j] = fmaxf(sv.of(root[j]), fminf(root[j] * 0x1p+100f, 0x1p-9f));     // (roots are 2^-75 at least: 2^-9, or zero of zero)
        store_8bit<PAST, FULL>(static_cast<uint8_t *>(of[kV]), i, end, y);
    } else {
        store_some<PAST, FULL>(static_cast<float *>(of[kM]), i, end, m);
        store_some<PAST, FULL>(static_cast<float *>(of[kV]), i, end, v);
    }
}

template <typename TW, typename TG, bool EIGHT, bool COPY, bool PAST>
__global__ void __launch_bounds__(kStepThreads)
k_adamw(StepArgs<EIGHT, COPY> a) {
    using Args = StepArgs<EIGHT, COPY>;
    using Shape = StepShape<TW, EIGHT>;
    const StepPlan &p = a.plan;
    const int which = tensor_of<Args::kTensors>(a.first, p.count, blockIdx.x);
    const uint32_t first = a.first[which], next = which + 1 < p.count ? a.first[which + 1] : p.groups;
    const uint32_t rest = a.rest[which];
    const int shift = EIGHT ? 0 : static_cast<int>(rest >> 24);
    const int64_t end = int64_t(next - first - 1) * Shape::kGroup + static_cast<int>(rest & 0xFFFF) + 1 - shift;
    const int64_t group = int64_t(blockIdx.x - first) * Shape::kGroup - shift;
    void *of[Args::kPointers];
#pragma unroll
    for (int k = 0; k < Args::kPointers; ++k) of[k] = a.get(k, which);
    StepFactors f = p.factors[rest >> 16 & 0xFF];
    StepNumbers n{1.f, f.size, f.keep, p.beta1_f, p.beta2_f, p.new1, p.new2, p.root_by, p.eps, p.copy_type};
    if (p.grad_scale) {
        n.by = *p.grad_scale;
        if (!(fabsf(n.by) < __uint_as_float(0x7F800000u))) return;     // nothing is stepped by gradients whose norm is no number
    }
    if (p.step || p.lr_dev) {
        const int64_t t = p.step ? *p.step : a.plan.host_step;
        const int64_t step = t > 1 ? t : 1;
        set_factors(f, p.lr_dev ? static_cast<double>(*p.lr_dev) : p.lr, p.decay, p.beta1, step);
        n.size = f.size;
        n.keep = f.keep;
        n.root_by = debiased_root_by(p.beta2, step);
    }
    const int64_t base = group + static_cast<int>(threadIdx.x) * Shape::kElems;
    const bool full = group >= 0 && group + Shape::kGroup <= end;
    bool lines = false;
    if constexpr (EIGHT && PAST) lines = (reinterpret_cast<uint64_t>(of[kM]) | reinterpret_cast<uint64_t>(of[kV])) % kLine == 0;
    if (full && lines) step_group<TW, TG, EIGHT, COPY, PAST, true, true>(n, of, base, end);
    else if (full) step_group<TW, TG, EIGHT, COPY, PAST, true, false>(n, of, base, end);
    else step_group<TW, TG, EIGHT, COPY, PAST, false, false>(n, of, base, end);
}

// What a launch of the norm knows: the tensors' gradients, their first chunks and the elements of their last ones.
constexpr int kNormTensors = 250;
struct NormEnd {
    float mul, most;
    float *norm, *scale;
};
struct GradNormArgs {
    double *parts;                       // [workgroups] sums of squares
    uint32_t *done;                      // workgroups that have theirs; zero between launches
    NormEnd end;
    uint32_t chunks;                     // of all tensors
    int32_t count, add;                  // add: workgroups that have a sum of the launch before
    const void *grad[kNormTensors];
    uint32_t first[kNormTensors];
    uint32_t rest[kNormTensors];         // the last chunk's elements less one, shift << 24
};
static_assert(sizeof(GradNormArgs) <= kArgBytes, "a launch's arguments");

constexpr int kNormElems = 32;                         // of a thread and chunk
constexpr int kNormChunk = kBlock * kNormElems;
constexpr int kJoinParts = kWave;                      // so many workgroups at most: the last of them ends the norm

// The norm of the sum of squares, and the factor that brings it to `most`.
__device__ __forceinline__ void end_norm(const NormEnd &e, double squares) {
    const float found = static_cast<float>(e.mul * sqrt(squares));
    if (e.norm) *e.norm = found;
    if (!e.scale) return;
    // (the reciprocal of a norm below 2^-126 may be infinite, and that of one above 2^126 has lost bits)
    const float share = found >= 0x1p-126f && found <= 0x1p+126f ? e.most * (1.0f / found) : e.most / found;
    *e.scale = found < __uint_as_float(0x7F800000u) ? e.mul * fminf(share, 1.f) : __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// A sum of squares outside this range may have lost terms at either end of 32 bits' range (or is zero, or no number).
__device__ __forceinline__ bool odd_sum(float sum) { return !(sum >= 0x1p-90f && sum <= 0x1p+120f); }

// Every workgroup's sum of squares.  Sixteen squares are added in 32 bits, which is enough where none of them leaves its range; others, and all sums of sums, have 64.
// JOIN: the last workgroup to be done adds the parts, in their order, and ends the norm.
template <typename T, bool JOIN, bool PAST>
__global__ void __launch_bounds__(kBlock)
k_grad_norm(GradNormArgs a) {
    __shared__ double lds[kWavesPerBlock];
    double all = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const int which = tensor_of<kNormTensors>(a.first, a.count, chunk);
        const uint32_t first = a.first[which], next = which + 1 < a.count ? a.first[which + 1] : a.chunks;
        const int shift = static_cast<int>(a.rest[which] >> 24);
        const int64_t end = int64_t(next - first - 1) * kNormChunk + static_cast<int>(a.rest[which] & 0xFFFF) + 1 - shift;
        const int64_t base = int64_t(chunk - first) * kNormChunk - shift;
        const T *grad = static_cast<const T *>(a.grad[which]);
        constexpr int V = Vec<T>::kLen, kLoads = kNormElems / V;
        typename Some<T, V>::Whole raw[kLoads];
        if (base >= 0 && base + kNormChunk <= end) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) raw[k] = load_some<PAST, true, V>(grad, base + (k * kBlock + static_cast<int>(threadIdx.x)) * V, end);
        } else {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) raw[k] = load_some<PAST, false, V>(grad, base + (k * kBlock + static_cast<int>(threadIdx.x)) * V, end);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float sum = 0.f, most = 0.f;
#pragma unroll
            for (int k = half * kLoads / 2; k < (half + 1) * kLoads / 2; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float g = static_cast<float>(raw[k][j]);
                    sum = fmaf(g, g, sum);
                    most = fmaxf(most, fabsf(g));
                }
            if (odd_sum(sum) && (most > 0.f || sum != sum)) {
#pragma unroll
                for (int k = half * kLoads / 2; k < (half + 1) * kLoads / 2; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const double g = static_cast<double>(static_cast<float>(raw[k][j]));
                        all = fma(g, g, all);
                    }
            } else {
                all += static_cast<double>(sum);
            }
        }
    }
    all = wave_sum(all);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    all = 0.0;
#pragma unroll
    for (int k = 0; k < kWavesPerBlock; ++k) all += lds[k];
    if constexpr (JOIN) {
        // (the dies' L2s are not one another's: parts and their number go past them)
        uint32_t before = 0;
        if (threadIdx.x == 0) {
            __hip_atomic_store(a.parts + blockIdx.x, all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            before = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (__builtin_amdgcn_readfirstlane(static_cast<int>(before)) + 1 != static_cast<int>(gridDim.x)) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        all = threadIdx.x < gridDim.x ? __hip_atomic_load(a.parts + threadIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        all = wave_sum(all);
        if (threadIdx.x == 0) {
            __hip_atomic_store(a.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            end_norm(a.end, all);
        }
    } else if (threadIdx.x == 0) {
        a.parts[blockIdx.x] = all + (static_cast<int>(blockIdx.x) < a.add ? a.parts[blockIdx.x] : 0.0);
    }
}

constexpr int kEndThreads = 1024;
__global__ void __launch_bounds__(kEndThreads)
k_grad_norm_end(const double *parts, int num, NormEnd e) {
    __shared__ double lds[kEndThreads / kWave];
    double all = 0.0;
    for (int p = static_cast<int>(threadIdx.x); p < num; p += kEndThreads) all += parts[p];
    all = wave_sum(all);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    all = wave_sum(threadIdx.x < kEndThreads / kWave ? lds[threadIdx.x] : 0.0);
    if (threadIdx.x == 0) end_norm(e, all);
}

int type_size(int32_t dtype) { return dtype == MQG_F32 ? 4 : 2; }

template <typename TW, typename TG, bool EIGHT, bool COPY>
int launch_step(mqg_ctx *ctx, const StepArgs<EIGHT, COPY> &a, bool past, hipStream_t s) {
    if (past) MQG_LAUNCH(ctx, "k_adamw", s, (k_adamw<TW, TG, EIGHT, COPY, true><<<a.plan.groups, kStepThreads, 0, s>>>(a)));
    else MQG_LAUNCH(ctx, "k_adamw", s, (k_adamw<TW, TG, EIGHT, COPY, false><<<a.plan.groups, kStepThreads, 0, s>>>(a)));
    return MQG_OK;
}

// The tensors of one kind, a launch's at a time.
template <typename TW, typename TG, bool EIGHT, bool COPY, typename Wanted>
int step_tensors(mqg_ctx *ctx, const mqg_param *params, int32_t num, const StepPlan &plan, bool past, Wanted wanted, hipStream_t s) {
    using Args = StepArgs<EIGHT, COPY>;
    constexpr int64_t kGroup = StepShape<TW, EIGHT>::kGroup;
    Args a;
    a.plan = plan;
    a.plan.count = 0;
    a.plan.groups = 0;
    int factors = 0;
    auto launch = [&]() -> int {
        if (a.plan.count == 0) return MQG_OK;
        const int rc = launch_step<TW, TG, EIGHT, COPY>(ctx, a, past, s);
        a.plan.count = factors = 0;
        a.plan.groups = 0;
        return rc;
    };
    for (int32_t i = 0; i < num; ++i) {
        const mqg_param &p = params[i];
        if (!wanted(p)) continue;
        for (int64_t done = 0; done < p.numel;) {          // (parts are whole workgroups, and so whole blocks of 8-bit moments)
            int f = 0;
            while (f < factors && (a.plan.factors[f].lr_scale != p.lr_scale || a.plan.factors[f].decay_scale != p.decay_scale)) ++f;
            if (a.plan.count == Args::kTensors || f == kFactors || a.plan.groups >= kMostElems / kGroup) {
                const int rc = launch();
                if (rc != MQG_OK) return rc;
                f = 0;
            }
            if (f == factors) {
                a.plan.factors[f].lr_scale = p.lr_scale;
                a.plan.factors[f].decay_scale = p.decay_scale;
                set_factors(a.plan.factors[f], plan.lr, plan.decay, plan.beta1, plan.host_step);
                ++factors;
            }
            const int64_t part = std::min(p.numel - done, (kMostElems / kGroup - a.plan.groups) * kGroup);
            const int at = a.plan.count++;
            a.set(kWeight, at, static_cast<TW *>(p.weight) + done);
            a.set(kGrad, at, static_cast<const TG *>(p.grad) + done);
            a.set(kM, at, static_cast<char *>(p.m) + done * (EIGHT ? 1 : 4));
            a.set(kV, at, static_cast<char *>(p.v) + done * (EIGHT ? 1 : 4));
            if constexpr (COPY) a.set(Args::kCopy, at, static_cast<char *>(p.copy) + done * type_size(p.copy_type));
            if constexpr (EIGHT) {
                a.set(Args::kMScale, at, p.m_scale + done / MQG_ADAMW_BLOCK);
                a.set(Args::kVScale, at, p.v_scale + done / MQG_ADAMW_BLOCK);
            }
            a.first[at] = a.plan.groups;
            const int shift = EIGHT ? 0 : line_shift(static_cast<TW *>(p.weight) + done);
            a.rest[at] = static_cast<uint32_t>((part + shift - 1) % kGroup) | static_cast<uint32_t>(f) << 16 | static_cast<uint32_t>(shift) << 24;
            a.plan.groups += static_cast<uint32_t>(ceil_div(part + shift, kGroup));
            done += part;
        }
    }
    return launch();
}

}  // namespace

int run_grad_norm(mqg_ctx *ctx, const mqg_param *params, int32_t num, float mul, float most, float *norm, float *scale, hipStream_t s) {
    GradNormArgs a;
    a.parts = ctx->norm_parts;
    a.done = reinterpret_cast<uint32_t *>(ctx->norm_parts + kGradNormParts);
    a.end = {mul, most, norm, scale};
    // Tensors of one type that one launch takes need no second one if they are few.
    int64_t wanted = 0, bytes = 0, all_chunks = 0;
    int types = 0;
    for (int32_t type : {MQG_F32, MQG_F16, MQG_BF16}) {
        bool met = false;
        for (int32_t i = 0; i < num; ++i) {
            const mqg_param &p = params[i];
            if (!p.grad || p.numel == 0 || p.grad_type != type) continue;
            met = true;
            ++wanted;
            bytes += p.numel * type_size(type);
            all_chunks += ceil_div(p.numel + line_shift(static_cast<const char *>(p.grad)) / type_size(type), kNormChunk);
        }
        types += met;
    }
    const bool join = types == 1 && wanted <= kNormTensors && all_chunks <= kJoinParts, past = bytes >= kNormPastBytes;
    int parts = 0;
    for (int32_t type : {MQG_F32, MQG_F16, MQG_BF16}) {
        a.count = 0;
        a.chunks = 0;
        auto launch = [&]() -> int {
            if (a.count == 0) return MQG_OK;
            const int grid = static_cast<int>(std::min<int64_t>(a.chunks, kGradNormParts));
            a.add = parts;
#define MQG_GO(T)                                                                                                  \
    do {                                                                                                           \
        if (join) MQG_LAUNCH(ctx, "k_grad_norm", s, (k_grad_norm<T, true, false><<<grid, kBlock, 0, s>>>(a)));       \
        else if (past) MQG_LAUNCH(ctx, "k_grad_norm", s, (k_grad_norm<T, false, true><<<grid, kBlock, 0, s>>>(a)));  \
        else MQG_LAUNCH(ctx, "k_grad_norm", s, (k_grad_norm<T, false, false><<<grid, kBlock, 0, s>>>(a)));           \
    } while (0)
            if (type == MQG_F16) MQG_GO(F16);
            else if (type == MQG_BF16) MQG_GO(BF16);
            else MQG_GO(float);
#undef MQG_GO
            parts = std::max(parts, grid);
            a.count = 0;
            a.chunks = 0;
            return MQG_OK;
        };
        for (int32_t i = 0; i < num; ++i) {
            const mqg_param &p = params[i];
            if (!p.grad || p.grad_type != type) continue;
            for (int64_t done = 0; done < p.numel;) {
                if (a.count == kNormTensors || a.chunks >= kMostElems / kNormChunk) {
                    const int rc = launch();
                    if (rc != MQG_OK) return rc;
                }
                const int64_t part = std::min(p.numel - done, (kMostElems / kNormChunk - a.chunks) * kNormChunk);
                const char *grad = static_cast<const char *>(p.grad) + done * type_size(type);
                const int shift = line_shift(grad) / type_size(type);
                a.grad[a.count] = grad;
                a.rest[a.count] = static_cast<uint32_t>((part + shift - 1) % kNormChunk) | static_cast<uint32_t>(shift) << 24;
                a.first[a.count++] = a.chunks;
                a.chunks += static_cast<uint32_t>(ceil_div(part + shift, kNormChunk));
                done += part;
            }
        }
        const int rc = launch();
        if (rc != MQG_OK) return rc;
    }
    if (!join) MQG_LAUNCH(ctx, "k_grad_norm_end", s, (k_grad_norm_end<<<1, kEndThreads, 0, s>>>(ctx->norm_parts, parts, a.end)));
    return MQG_OK;
}

int run_adamw_step(mqg_ctx *ctx, const mqg_param *params, int32_t num, const mqg_adamw *plan, hipStream_t s) {
    StepPlan a = {};
    a.lr = plan->lr;
    a.decay = plan->weight_decay;
    a.beta1 = plan->beta1;
    a.beta2 = plan->beta2;
    a.host_step = std::max<int64_t>(plan->step, 1);
    a.beta1_f = static_cast<float>(plan->beta1);
    a.beta2_f = static_cast<float>(plan->beta2);
    a.new1 = static_cast<float>(1.0 - plan->beta1);
    a.new2 = static_cast<float>(1.0 - plan->beta2);
    a.root_by = debiased_root_by(plan->beta2, a.host_step);
    a.step = plan->step_dev;
    a.lr_dev = plan->lr_dev;
    a.grad_scale = plan->grad_scale_dev;
    a.eps = plan->eps < 0x1p-126 ? 0.f : static_cast<float>(plan->eps);
    // Tensors of the same types go together.  A kind: the types of weight and gradient, that of the moments, and that of the copy (3: none).
    auto kind_of = [](const mqg_param &p) { return ((p.weight_type * 3 + p.grad_type) * 2 + p.state_type) * 4 + (p.copy ? p.copy_type : 3); };
    constexpr int kKinds = 3 * 3 * 2 * 4;
    bool met[kKinds] = {};
    int64_t bytes = 0;
    for (int32_t i = 0; i < num; ++i) {
        const mqg_param &p = params[i];
        if (!p.grad || p.numel == 0) continue;
        met[kind_of(p)] = true;
        bytes += p.numel * (2 * type_size(p.weight_type) + type_size(p.grad_type) + (p.copy ? type_size(p.copy_type) : 0) + (p.state_type == MQG_STATE_E4M3 ? 4 : 16));
    }
    const bool past = bytes >= kStepPastBytes;
    for (int kind = 0; kind < kKinds; ++kind) {
        if (!met[kind]) continue;
        auto wanted = [&](const mqg_param &p) { return p.grad && p.numel > 0 && kind_of(p) == kind; };
        const bool eight = (kind / 4) % 2 != 0, copy = kind % 4 != 3;
        a.copy_type = kind % 4;
        auto go = [&](auto weight, auto grad) -> int {
            using TW = decltype(weight);
            using TG = decltype(grad);
            if (eight) return copy ? step_tensors<TW, TG, true, true>(ctx, params, num, a, past, wanted, s) : step_tensors<TW, TG, true, false>(ctx, params, num, a, past, wanted, s);
            return copy ? step_tensors<TW, TG, false, true>(ctx, params, num, a, past, wanted, s) : step_tensors<TW, TG, false, false>(ctx, params, num, a, past, wanted, s);
        };
        auto of_grads = [&](auto weight) -> int {
            const int type = (kind / 8) % 3;
            return type == MQG_F16 ? go(weight, F16()) : type == MQG_BF16 ? go(weight, BF16()) : go(weight, float());
        };
        const int type = kind / 24;
        const int rc = type == MQG_F16 ? of_grads(F16()) : type == MQG_BF16 ? of_grads(BF16()) : of_grads(float());
        if (rc != MQG_OK) return rc;
    }
    return MQG_OK;
}

}  // namespace mqg
