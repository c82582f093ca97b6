// The norm of all gradients, and the AdamW step of many tensors in a launch, with moments in 32 bits or in 8.
//
//   norm   n = mul sqrt(sum over all g^2),  scale = mul min(1, most / n)
//   step   g' = scale g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
//          w = (1 - lr decay) w - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
//   8 bits m and sqrt(v) of 128 elements in order as e4m3 values times a scale that is the block's own: the largest of each keeps 32 bits.  The root instead of
//          v itself: e4m3 reaches down to 2^-18 of its largest value, which is 2^-36 of v.  A root above zero that would round to zero becomes the least
//          value above it, so that no moment is divided by epsilon alone.
//
// Both are bound by memory: what is read is read once, what is written is written once.  The tensors' addresses and sizes come with the launch,
// kTensors at a time, so that nothing is copied to the device beforehand; a workgroup finds its tensor by a comparison in every lane.
#include <algorithm>
#include <cmath>
#include <vector>

#include "common.h"
#include "layer_types.h"

namespace mqg {
namespace {

constexpr int kTensors = 48;             // of a launch of the step: 72 + 4 bytes each of the 4 KB that a launch's arguments have
constexpr int kNormTensors = 64;         // of a launch of the norm, one a lane
constexpr int64_t kMostElems = int64_t(1) << 31;       // of a launch; longer tensors go in parts

// Which of `count` tensors workgroup `group` belongs to: the last that begins at it or before.
__device__ __forceinline__ int tensor_of(const uint32_t *first, int count, uint32_t group) {
    const int lane = lane_id();
    const bool before = lane < count && first[lane] <= group;
    return __builtin_amdgcn_readfirstlane(popc64(ballot64(before)) - 1);
}

// beta^t for t >= 1, by squaring
__host__ __device__ __forceinline__ double power(double beta, int64_t t) {
    double all = 1.0;
    for (double p = beta; t > 0; t >>= 1, p *= p)
        if (t & 1) all *= p;
    return all;
}

struct StepTensor {
    void *weight;
    const void *grad;
    void *copy, *m, *v;
    float *m_scale, *v_scale;
    int64_t numel;
    float lr_scale, decay_scale;
};
struct StepArgs {
    uint32_t first[kTensors];            // the tensors' first workgroups
    StepTensor of[kTensors];
    double lr, decay, beta1, beta2;
    double debias1, debias2;             // 1 - beta^t, where the host knows t
    const int64_t *step;                 // else t
    const float *lr_dev, *grad_scale;
    float eps;
    int32_t count, copy_type;            // copy_type: -1 for none
};

// N elements of a tensor from i on as 32-bit numbers; zeros past its end
template <typename T, int N>
__device__ __forceinline__ void load_some(const T *p, int64_t i, int64_t end, float (&out)[N]) {
    typedef T Some __attribute__((ext_vector_type(N)));
    typedef Some Any __attribute__((aligned(sizeof(T))));
    if (i + N <= end) {
        const Some v = *reinterpret_cast<const Any *>(p + i);
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = static_cast<float>(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = i + j < end ? static_cast<float>(p[i + j]) : 0.f;
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T *p, int64_t i, int64_t end, const float (&in)[N]) {
    typedef T Some __attribute__((ext_vector_type(N)));
    typedef Some Any __attribute__((aligned(sizeof(T))));
    if (i + N <= end) {
        Some v;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = static_cast<T>(in[j]);
        *reinterpret_cast<Any *>(p + i) = v;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i + j < end) p[i + j] = static_cast<T>(in[j]);
    }
}

// Eight e4m3 values
__device__ __forceinline__ void load_8bit(const uint8_t *p, int64_t i, int64_t end, float (&out)[8]) {
    uint32_t w[2] = {0, 0};
    if (i + 8 <= end) {
        typedef uint32_t Two __attribute__((ext_vector_type(2)));
        typedef Two AnyTwo __attribute__((aligned(1)));
        const Two v = *reinterpret_cast<const AnyTwo *>(p + i);
        w[0] = v[0];
        w[1] = v[1];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < end) w[j / 4] |= static_cast<uint32_t>(p[i + j]) << (8 * (j % 4));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        out[4 * k] = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w[k]), 0);
        out[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w[k]), 1);
        out[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w[k]), 2);
        out[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w[k]), 3);
    }
}
__device__ __forceinline__ void store_8bit(uint8_t *p, int64_t i, int64_t end, const uint32_t (&w)[2]) {
    if (i + 8 <= end) {
        typedef uint32_t Two __attribute__((ext_vector_type(2)));
        typedef Two AnyTwo __attribute__((aligned(1)));
        Two v;
        v[0] = w[0];
        v[1] = w[1];
        *reinterpret_cast<AnyTwo *>(p + i) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < end) p[i + j] = static_cast<uint8_t>(w[j / 4] >> (8 * (j % 4)));
    }
}
// Words whose zero bytes are ones where the value is above zero
__device__ __forceinline__ void lift(const float (&v)[8], uint32_t (&w)[2]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (v[j] > 0.f && !((w[j / 4] >> (8 * (j % 4))) & 0xFF)) w[j / 4] |= 1u << (8 * (j % 4));
}

constexpr int kStepElems = 8;                              // of a thread
constexpr int kStepGroup = kBlock * kStepElems;            // of a workgroup: 16 blocks of 8-bit moments
constexpr int kScaleLanes = MQG_ADAMW_BLOCK / kStepElems;  // that share a scale

template <typename TW, typename TG, bool EIGHT>
__global__ void __launch_bounds__(kBlock)
k_adamw(StepArgs a) {
    float by = 1.f;
    if (a.grad_scale) {
        by = *a.grad_scale;
        if (!(fabsf(by) < __uint_as_float(0x7F800000u))) return;       // nothing is stepped by gradients whose norm is no number
    }
    const int which = tensor_of(a.first, a.count, blockIdx.x);
    const StepTensor &t = a.of[which];
    const int64_t end = t.numel;
    const int64_t i = int64_t(blockIdx.x - a.first[which]) * kStepGroup + threadIdx.x * kStepElems;
    double debias1 = a.debias1, debias2 = a.debias2;
    if (a.step) {
        const int64_t step = *a.step;
        debias1 = 1.0 - power(a.beta1, step > 1 ? step : 1);
        debias2 = 1.0 - power(a.beta2, step > 1 ? step : 1);
    }
    const double lr = (a.lr_dev ? static_cast<double>(*a.lr_dev) : a.lr) * t.lr_scale;
    const float keep = static_cast<float>(1.0 - lr * (a.decay * t.decay_scale));
    const float size = static_cast<float>(lr / debias1);
    const float root_by = static_cast<float>(1.0 / sqrt(debias2));
    const float beta1 = static_cast<float>(a.beta1), beta2 = static_cast<float>(a.beta2);
    const float new1 = static_cast<float>(1.0 - a.beta1), new2 = static_cast<float>(1.0 - a.beta2);

    float w[8], g[8], m[8], v[8];
    load_some(static_cast<const TG *>(t.grad), i, end, g);
    load_some(static_cast<const TW *>(t.weight), i, end, w);
    const int64_t block = i / MQG_ADAMW_BLOCK;
    if constexpr (EIGHT) {
        load_8bit(static_cast<const uint8_t *>(t.m), i, end, m);
        load_8bit(static_cast<const uint8_t *>(t.v), i, end, v);
        const float ms = i < end ? t.m_scale[block] : 0.f, vs = i < end ? t.v_scale[block] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] *= ms;
            v[j] *= vs;
            v[j] *= v[j];
        }
    } else {
        load_some(static_cast<const float *>(t.m), i, end, m);
        load_some(static_cast<const float *>(t.v), i, end, v);
    }
    float root[8];
    uint32_t most_m = 0, most_root = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] *= by;
        m[j] = fmaf(beta1, m[j], new1 * g[j]);
        v[j] = fmaf(beta2, v[j], new2 * g[j] * g[j]);
        root[j] = sqrtf(v[j]);
        const float under = fmaf(root[j], root_by, a.eps);
        const float step = under == 0.f ? 0.f : size * m[j] / under;
        w[j] = fmaf(w[j], keep, -step);
        most_m = max_u32(most_m, __float_as_uint(m[j]) & 0x7FFFFFFFu);
        most_root = max_u32(most_root, __float_as_uint(root[j]) & 0x7FFFFFFFu);
    }
    store_some(static_cast<TW *>(t.weight), i, end, w);
    if (t.copy) {
        if (a.copy_type == MQG_F16) store_some(static_cast<F16 *>(t.copy), i, end, w);
        else if (a.copy_type == MQG_BF16) store_some(static_cast<BF16 *>(t.copy), i, end, w);
        else store_some(static_cast<float *>(t.copy), i, end, w);
    }
    if constexpr (EIGHT) {
        const Scale sm = scale_of(lanes_max(most_m, kScaleLanes), 1.f, 448.f), sv = scale_of(lanes_max(most_root, kScaleLanes), 1.f, 448.f);
        if (threadIdx.x % kScaleLanes == 0 && i < end) {
            t.m_scale[block] = sm.scale;
            t.v_scale[block] = sv.scale;
        }
        uint32_t q[2];
        to_8bit(m, sm, MQG_Q_E4M3, q);
        store_8bit(static_cast<uint8_t *>(t.m), i, end, q);
        to_8bit(root, sv, MQG_Q_E4M3, q);
        lift(root, q);
        store_8bit(static_cast<uint8_t *>(t.v), i, end, q);
    } else {
        store_some(static_cast<float *>(t.m), i, end, m);
        store_some(static_cast<float *>(t.v), i, end, v);
    }
}

struct NormTensor {
    const void *grad;
    int64_t numel;
};
struct GradNormArgs {
    uint32_t first[kNormTensors];
    NormTensor of[kNormTensors];
    double *parts;                       // [workgroups] sums of squares
    uint32_t chunks;                     // of all tensors
    int32_t count, add;                  // add: workgroups that have a sum of the launch before
};

constexpr int kNormElems = 16;                         // of a thread and chunk
constexpr int kNormChunk = kBlock * kNormElems;

// A sum of squares outside this range may have lost terms at either end of 32 bits' range (or is zero, or no number).
__device__ __forceinline__ bool odd_sum(float sum) { return !(sum >= 0x1p-90f && sum <= 0x1p+120f); }

// Every workgroup's sum of squares.  Sixteen squares are added in 32 bits, which is enough where none of them leaves its range; others, and all sums of sums, have 64.
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_grad_norm(GradNormArgs a) {
    __shared__ double lds[kWavesPerBlock];
    double all = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const int which = tensor_of(a.first, a.count, chunk);
        const NormTensor &t = a.of[which];
        const int64_t base = int64_t(chunk - a.first[which]) * kNormChunk;
        float g[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) load_some(static_cast<const T *>(t.grad), base + (k * kBlock + threadIdx.x) * 8, t.numel, g[k]);
        float sum = 0.f, most = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum = fmaf(g[k][j], g[k][j], sum);
                most = fmaxf(most, fabsf(g[k][j]));
            }
        if (odd_sum(sum) && (most > 0.f || sum != sum)) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) all = fma(static_cast<double>(g[k][j]), static_cast<double>(g[k][j]), all);
        } else {
            all += static_cast<double>(sum);
        }
    }
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) all += __shfl_xor(all, off, kWave);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        all = static_cast<int>(blockIdx.x) < a.add ? a.parts[blockIdx.x] : 0.0;
#pragma unroll
        for (int k = 0; k < kWavesPerBlock; ++k) all += lds[k];
        a.parts[blockIdx.x] = all;
    }
}

// The norm of the parts' sum, and the factor that brings it to `most`.
__global__ void __launch_bounds__(kBlock)
k_grad_norm_end(const double *parts, int num, double mul, double most, float *norm, float *scale) {
    __shared__ double lds[kWavesPerBlock];
    double all = 0.0;
    for (int p = static_cast<int>(threadIdx.x); p < num; p += kBlock) all += parts[p];
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) all += __shfl_xor(all, off, kWave);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        all = 0.0;
#pragma unroll
        for (int k = 0; k < kWavesPerBlock; ++k) all += lds[k];
        const double n = mul * sqrt(all);
        const float found = static_cast<float>(n);
        if (norm) *norm = found;
        if (scale) *scale = found < __uint_as_float(0x7F800000u) ? static_cast<float>(n > most ? mul * (most / n) : mul) : __uint_as_float(0x7FC00000u);
    }
}

int type_size(int32_t dtype) { return dtype == MQG_F32 ? 4 : 2; }

template <bool EIGHT>
int launch_step(mqg_ctx *ctx, int32_t weight_type, int32_t grad_type, const StepArgs &a, uint32_t groups, hipStream_t s) {
#define MQG_GO(TW, TG) MQG_LAUNCH(ctx, "k_adamw", s, (k_adamw<TW, TG, EIGHT><<<groups, kBlock, 0, s>>>(a)))
#define MQG_GRADS(TW)                              \
    if (grad_type == MQG_F16) MQG_GO(TW, F16);     \
    else if (grad_type == MQG_BF16) MQG_GO(TW, BF16); \
    else MQG_GO(TW, float);
    if (weight_type == MQG_F16) {
        MQG_GRADS(F16)
    } else if (weight_type == MQG_BF16) {
        MQG_GRADS(BF16)
    } else {
        MQG_GRADS(float)
    }
#undef MQG_GRADS
#undef MQG_GO
    return MQG_OK;
}

}  // namespace

int run_grad_norm(mqg_ctx *ctx, const mqg_param *params, int32_t num, float mul, float most, float *norm, float *scale, hipStream_t s) {
    int parts = 0;
    for (int32_t type : {MQG_F32, MQG_F16, MQG_BF16}) {
        GradNormArgs a;
        a.parts = ctx->norm_parts;
        a.count = 0;
        int64_t chunks = 0;
        auto launch = [&]() -> int {
            if (a.count == 0) return MQG_OK;
            const int grid = static_cast<int>(std::min<int64_t>(chunks, kGradNormParts));
            a.chunks = static_cast<uint32_t>(chunks);
            a.add = parts;
            if (type == MQG_F16) MQG_LAUNCH(ctx, "k_grad_norm", s, (k_grad_norm<F16><<<grid, kBlock, 0, s>>>(a)));
            else if (type == MQG_BF16) MQG_LAUNCH(ctx, "k_grad_norm", s, (k_grad_norm<BF16><<<grid, kBlock, 0, s>>>(a)));
            else MQG_LAUNCH(ctx, "k_grad_norm", s, (k_grad_norm<float><<<grid, kBlock, 0, s>>>(a)));
            parts = std::max(parts, grid);
            a.count = 0;
            chunks = 0;
            return MQG_OK;
        };
        for (int32_t i = 0; i < num; ++i) {
            const mqg_param &p = params[i];
            if (!p.grad || p.grad_type != type) continue;
            for (int64_t done = 0; done < p.numel;) {
                if (a.count == kNormTensors || chunks == kMostElems / kNormChunk) {
                    int rc = launch();
                    if (rc != MQG_OK) return rc;
                }
                const int64_t part = std::min(p.numel - done, (kMostElems / kNormChunk - chunks) * kNormChunk);
                a.first[a.count] = static_cast<uint32_t>(chunks);
                a.of[a.count++] = {static_cast<const char *>(p.grad) + done * type_size(type), part};
                chunks += ceil_div(part, kNormChunk);
                done += part;
            }
        }
        int rc = launch();
        if (rc != MQG_OK) return rc;
    }
    MQG_LAUNCH(ctx, "k_grad_norm_end", s, (k_grad_norm_end<<<1, kBlock, 0, s>>>(ctx->norm_parts, parts, mul, most, norm, scale)));
    return MQG_OK;
}

int run_adamw_step(mqg_ctx *ctx, const mqg_param *params, int32_t num, const mqg_adamw *plan, hipStream_t s) {
    StepArgs a;
    a.lr = plan->lr;
    a.decay = plan->weight_decay;
    a.beta1 = plan->beta1;
    a.beta2 = plan->beta2;
    a.debias1 = a.debias2 = 1.0;
    if (!plan->step_dev) {
        a.debias1 = 1.0 - power(plan->beta1, plan->step);
        a.debias2 = 1.0 - power(plan->beta2, plan->step);
    }
    a.step = plan->step_dev;
    a.lr_dev = plan->lr_dev;
    a.grad_scale = plan->grad_scale_dev;
    a.eps = static_cast<float>(plan->eps);
    // Tensors of the same types go together.
    auto key_of = [](const mqg_param &p) { return ((p.weight_type * 3 + p.grad_type) * 2 + p.state_type) * 4 + (p.copy ? p.copy_type : 3); };
    uint64_t left[2] = {0, 0};
    for (int32_t i = 0; i < num; ++i)
        if (params[i].grad && params[i].numel > 0) left[key_of(params[i]) >> 6] |= uint64_t(1) << (key_of(params[i]) & 63);
    for (int key = 0; key < 72; ++key) {
        if (!((left[key >> 6] >> (key & 63)) & 1)) continue;
        a.count = 0;
        a.copy_type = key % 4;
        const bool eight = (key / 4) % 2 != 0;
        const int32_t grad_type = (key / 8) % 3, weight_type = key / 24;
        int64_t groups = 0;
        auto launch = [&]() -> int {
            if (a.count == 0) return MQG_OK;
            const int rc = eight ? launch_step<true>(ctx, weight_type, grad_type, a, static_cast<uint32_t>(groups), s)
                                 : launch_step<false>(ctx, weight_type, grad_type, a, static_cast<uint32_t>(groups), s);
            a.count = 0;
            groups = 0;
            return rc;
        };
        for (int32_t i = 0; i < num; ++i) {
            const mqg_param &p = params[i];
            if (!p.grad || p.numel == 0 || key_of(p) != key) continue;
            for (int64_t done = 0; done < p.numel;) {      // (parts are whole workgroups, and so whole blocks of 8-bit moments)
                if (a.count == kTensors || groups == kMostElems / kStepGroup) {
                    int rc = launch();
                    if (rc != MQG_OK) return rc;
                }
                const int64_t part = std::min(p.numel - done, (kMostElems / kStepGroup - groups) * kStepGroup);
                auto at = [&](void *q, int64_t bytes) { return q ? static_cast<char *>(q) + done * bytes : nullptr; };
                const int64_t block = done / MQG_ADAMW_BLOCK, state = eight ? 1 : 4;
                a.first[a.count] = static_cast<uint32_t>(groups);
                a.of[a.count++] = {at(p.weight, type_size(weight_type)), at(const_cast<void *>(p.grad), type_size(grad_type)), at(p.copy, type_size(p.copy_type)),
                                   at(p.m, state), at(p.v, state), eight ? p.m_scale + block : nullptr, eight ? p.v_scale + block : nullptr,
                                   part, p.lr_scale, p.decay_scale};
                groups += ceil_div(part, kStepGroup);
                done += part;
            }
        }
        int rc = launch();
        if (rc != MQG_OK) return rc;
    }
    return MQG_OK;
}

}  // namespace mqg
