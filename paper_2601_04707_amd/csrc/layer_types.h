// Element types, 16-byte vectors, wavefront reductions and the way to 8 bits of the kernels of a layer (norm.hip, layer_norm.hip, aggregate_q8.hip, orthogonal.hip,
// adamw.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.h"
#include "mqg.h"

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
template <bool PAST = false, typename T>
__device__ __forceinline__ typename Vec<T>::Whole load_span(const T *row, const Span<Vec<T>::kLen> &at, int dim) {
    constexpr int V = Vec<T>::kLen;
    typename Vec<T>::Whole v;
    if (dim >= V) {
        if constexpr (PAST) v = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::Any *>(row + at.base));
        else v = *reinterpret_cast<const typename Vec<T>::Any *>(row + at.base);
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

// What a lane and the one 16 (32) lanes from it have, the lower one's first, in both of them.
struct Pair {
    uint32_t x, y;
};
__device__ __forceinline__ Pair swap_rows(uint32_t v) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return {p[0], p[1]};
}
__device__ __forceinline__ Pair swap_halves(uint32_t v) {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return {p[0], p[1]};
}

// Sum over `width` neighbouring lanes (a power of two, the same in all lanes of the wavefront), the same in each of them:
// the two halves of every step are added in either order, so no lane rounds otherwise than another.
__device__ __forceinline__ float lanes_sum(float v, int width) {
    if (width > 1) v += dpp_f32<0xB1>(v);                  // lanes 1 0 3 2 of every four
    if (width > 2) v += dpp_f32<0x4E>(v);                  // lanes 2 3 0 1
    if (width > 4) v += dpp_f32<0x141>(v);                 // a half row of eight, mirrored
    if (width > 8) v += dpp_f32<0x140>(v);                 // a row of 16, mirrored
    if (width > 16) {
        const Pair p = swap_rows(__float_as_uint(v));
        v = __uint_as_float(p.x) + __uint_as_float(p.y);
    }
    if (width > 32) {
        const Pair p = swap_halves(__float_as_uint(v));
        v = __uint_as_float(p.x) + __uint_as_float(p.y);
    }
    return v;
}
__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int width) {
    if (width > 1) v = max_u32(v, dpp_u32<0xB1>(v));
    if (width > 2) v = max_u32(v, dpp_u32<0x4E>(v));
    if (width > 4) v = max_u32(v, dpp_u32<0x141>(v));
    if (width > 8) v = max_u32(v, dpp_u32<0x140>(v));
    if (width > 16) {
        const Pair p = swap_rows(v);
        v = max_u32(p.x, p.y);
    }
    if (width > 32) {
        const Pair p = swap_halves(v);
        v = max_u32(p.x, p.y);
    }
    return v;
}

// How a group is taken to 8 bits, from z = s w and the row's r, y = z r.  Values and scale have r in common, so q = z / (max|z| / top) has two roundings before
// its own and r's is none of them (of a million e4m3 values 0.4 to 0.7 are the neighbour of the one that the formula has in 64 bits, of int8 1.5 to 2; of y divided
// by its scale in 32 bits 0.7 to 0.9 and 2 to 2.2); where that quotient would leave 32 bits' range, or the scale is the least one, q = y / scale.
// most: the largest |z|'s bit pattern (patterns of absolute values order as the values do, with infinity and NaN above all others): a group that
// holds a value that is not finite has the scale NaN, so that all its values read NaN.
struct Scale {
    float scale, by, div;             // q = (z by) / div
};
__device__ __forceinline__ Scale scale_of(uint32_t most, float r, float top) {
    const float t = __uint_as_float(most) / top, scale = t * r;
    if (!(scale < __uint_as_float(0x7F800000u))) {
        const float nan = __uint_as_float(0x7FC00000u);
        return {nan, nan, nan};
    }
    if (!(scale > 0x1p-126f)) return {0x1p-126f, r, 0x1p-126f};
    return t > 0x1p-100f ? Scale{scale, 1.f, t} : Scale{scale, r, scale};
}

// V quotients in 8 bits, four to a word.  number: their scale is one
template <int V>
__device__ __forceinline__ void pack_8bit(const float (&y)[V], bool number, int q_type, uint32_t (&w)[V / 4]) {
    if (q_type == MQG_Q_E4M3) {
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false);
            w[k] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2], y[4 * k + 3], p, true));
        }
    } else {
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            w[k] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = number ? static_cast<int>(rintf(y[4 * k + j])) : 0;
                w[k] |= (static_cast<uint32_t>(v) & 0xFFu) << (8 * j);
            }
        }
    }
}
// V values in 8 bits
template <int V>
__device__ __forceinline__ void to_8bit(const float (&z)[V], const Scale &s, int q_type, uint32_t (&w)[V / 4]) {
    const float inv = 1.0f / s.div;
    float y[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {                          // the quotient by the reciprocal, and its remainder's
        const float num = z[j] * s.by, quot = num * inv;
        y[j] = fmaf(fmaf(-quot, s.div, num), inv, quot);
    }
    pack_8bit(y, s.scale == s.scale, q_type, w);
}

}  // namespace mqg
