// Element types, 16-byte vectors and wavefront reductions of the kernels of a layer (norm.hip, aggregate_q8.hip, orthogonal.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.h"

namespace mqg {

using F16 = _Float16;
using BF16 = __bf16;

// 16 bytes of elements at any address that an element may have: the card's loads and stores of 16 bytes need no more.
template <typename T>
struct Vec {
    static constexpr int kLen = 16 / static_cast<int>(sizeof(T));
    typedef T Whole __attribute__((ext_vector_type(kLen)));
    typedef Whole Any __attribute__((aligned(sizeof(T))));
};

// Vector number i of a row of dim elements as 32-bit numbers, zeros past its end; nothing outside the row is read.
template <typename T>
__device__ __forceinline__ void load_vec(const T *row, int i, int dim, float (&out)[Vec<T>::kLen]) {
    constexpr int V = Vec<T>::kLen;
    if ((i + 1) * V <= dim) {
        const typename Vec<T>::Whole v = *reinterpret_cast<const typename Vec<T>::Any *>(row + i * V);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = static_cast<float>(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = i * V + j < dim ? static_cast<float>(row[i * V + j]) : 0.f;
    }
}

// The same vector of a row that is written: rounded once, to nearest even; nothing outside the row is written.
template <typename T>
__device__ __forceinline__ void store_vec(T *row, int i, int dim, const float (&in)[Vec<T>::kLen]) {
    constexpr int V = Vec<T>::kLen;
    if ((i + 1) * V <= dim) {
        typename Vec<T>::Whole v;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = static_cast<T>(in[j]);
        *reinterpret_cast<typename Vec<T>::Any *>(row + i * V) = v;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (i * V + j < dim) row[i * V + j] = static_cast<T>(in[j]);
    }
}

// Vector number i of a row of dim elements without a branch on the lane (one element by element makes the wavefront wait for what it loads): the last
// vector of a row, and any past it, is the row's last V elements, of which the first `skip` are another lane's.
template <int V>
struct Span {
    int base, skip;
    __device__ __forceinline__ Span() = default;
    __device__ __forceinline__ Span(int i, int dim) {
        base = i * V < dim - V ? i * V : dim - V > 0 ? dim - V : 0;
        skip = i * V - base;
    }
    __device__ __forceinline__ bool mine(int j) const { return j >= skip; }
};
// Its elements as they lie; nothing outside the row is read, zeros past the end of a row of fewer than V.
template <typename T>
__device__ __forceinline__ typename Vec<T>::Whole load_span(const T *row, const Span<Vec<T>::kLen> &at, int dim) {
    constexpr int V = Vec<T>::kLen;
    typename Vec<T>::Whole v;
    if (dim >= V) {
        v = *reinterpret_cast<const typename Vec<T>::Any *>(row + at.base);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = j < dim ? row[j] : static_cast<T>(0.f);
    }
    return v;
}
// The elements that are its own, rounded once, to nearest even.  PAST: not to be kept in the caches (a template's argument: of a branch on it the
// compiler makes one store of the usual kind)
template <bool PAST, typename T>
__device__ __forceinline__ void store_span(T *row, const Span<Vec<T>::kLen> &at, int dim, const float (&in)[Vec<T>::kLen]) {
    constexpr int V = Vec<T>::kLen;
    if (at.skip == 0 && dim >= V) {
        typename Vec<T>::Whole v;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = static_cast<T>(in[j]);
        if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<typename Vec<T>::Any *>(row + at.base));
        else *reinterpret_cast<typename Vec<T>::Any *>(row + at.base) = v;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (at.mine(j) && at.base + j < dim) row[at.base + j] = static_cast<T>(in[j]);
    }
}
// The same columns of a [dim] vector of floats; null: ones
template <int V>
__device__ __forceinline__ void load_weight(const float *w, const Span<V> &at, int dim, float (&out)[V]) {
    if (w && dim >= V) {
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
            const typename Vec<float>::Whole x = *reinterpret_cast<const typename Vec<float>::Any *>(w + at.base + 4 * h);
#pragma unroll
            for (int j = 0; j < 4; ++j) out[4 * h + j] = x[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = !w ? 1.f : j < dim ? w[j] : 0.f;
    }
}

// A lane's register from the lane that the control word names, within rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}

// Sum over `width` neighbouring lanes (a power of two, the same in all lanes of the wavefront), the same in each of them:
// the two halves of every step are added in either order, so no lane rounds otherwise than another.
__device__ __forceinline__ float lanes_sum(float v, int width) {
    if (width > 1) v += dpp_f32<0xB1>(v);                  // lanes 1 0 3 2 of every four
    if (width > 2) v += dpp_f32<0x4E>(v);                  // lanes 2 3 0 1
    if (width > 4) v += dpp_f32<0x141>(v);                 // a half row of eight, mirrored
    if (width > 8) v += dpp_f32<0x140>(v);                 // a row of 16, mirrored
    if (width > 16) v += __shfl_xor(v, 16, kWave);
    if (width > 32) v += __shfl_xor(v, 32, kWave);
    return v;
}
__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int width) {
    if (width > 1) v = max_u32(v, dpp_u32<0xB1>(v));
    if (width > 2) v = max_u32(v, dpp_u32<0x4E>(v));
    if (width > 4) v = max_u32(v, dpp_u32<0x141>(v));
    if (width > 8) v = max_u32(v, dpp_u32<0x140>(v));
    if (width > 16) v = max_u32(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 16, kWave)));
    if (width > 32) v = max_u32(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 32, kWave)));
    return v;
}

}  // namespace mqg
