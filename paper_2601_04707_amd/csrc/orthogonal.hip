// Orthogonalising an update by Newton-Schulz products, and the weights' step around it.
//
//   U (n x k, n <= k, the transpose otherwise):  X = U / (|U|_F + eps), so that no singular value is above 1; then `steps` times
//       G = X X^T,   B = b G + c G G,   X <- a X + B X
//   which takes every singular value x to the odd polynomial a x + b x^3 + c x^5 and leaves the singular vectors as they are.
//   Step of the weights:  m <- beta m + g,  U = g + beta m (or m),  w <- w (1 - lr decay) - lr scale X.
//
// All three products are P Q^T of matrices whose rows are contiguous (G and B are symmetric, X is kept both ways), so there
// is one product kernel, with an epilogue for each.
//
// Numbers.  The iterates are held as two terms of f16, hi = f16(v), lo = f16(v - hi), 22 bits together, and a product is hi hi + hi lo +
// lo hi on the f16 matrix instructions with sums in 32 bits: what is left out, lo lo, is 2^-22 of it, so the error is that of a
// product in 32 bits at a third of the f16 rate (which is five times the rate of the card's 32-bit matrix instructions).
// Every matrix is stored times a power of two that puts the largest value it can have (known from the polynomial alone) just below f16's
// largest, which leaves 2^-39 of it for the smallest.
// Lines.  128 bytes of a row hold 32 values: their 32 high terms, then their 32 low ones.  A step of a product takes one line of every
// row of its tile, from memory to LDS without registers between; the 16-byte chunks of row r change places by an exclusive or with
// bits of r, so that the 16 rows that a wavefront reads together lie in different banks.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "layer_types.h"

namespace mqg {

namespace {

typedef F16 Half8 __attribute__((ext_vector_type(8)));
typedef F16 Half4 __attribute__((ext_vector_type(4)));
typedef float Float16v __attribute__((ext_vector_type(16)));

constexpr int kLine = 64;             // f16 of a line of 128 bytes
constexpr int kLineVals = 32;         // values of a line

__device__ __forceinline__ int chunk_place(int row, int chunk) { return chunk ^ (row & 7) ^ ((row >> 3) & 1); }

// Position of value v of a row: its high term's; the low term's is kLineVals further.
__device__ __forceinline__ int64_t term_at(int v) { return int64_t(v / kLineVals) * kLine + v % kLineVals; }

__device__ __forceinline__ void split(float v, F16 *hi, F16 *lo) {
    *hi = static_cast<F16>(v);
    *lo = static_cast<F16>(v - static_cast<float>(*hi));
}

// ---------------------------------------------------------------- the update and its norm

struct UpdateArgs {
    const void *grad;
    float *momentum;                  // null: the update is the gradient itself
    int64_t grad_row, grad_mat, mom_row, mom_mat;
    double *parts;                    // [mats x gridDim.x] sums of squares
    int32_t rows, cols, nesterov;
    float beta, eps;
};

// the update's value from the gradient and the new momentum
__device__ __forceinline__ float update_of(const UpdateArgs &a, float g, float m) { return !a.momentum ? g : a.nesterov ? g + a.beta * m : m; }

// m <- beta m + g, and every workgroup's share of |U|^2, in 64 bits: gradients of any size that 32 bits hold have a norm
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_muon_momentum(UpdateArgs a) {
    __shared__ double lds[kWavesPerBlock];
    const int mat = static_cast<int>(blockIdx.y);
    const T *grad = static_cast<const T *>(a.grad) + mat * a.grad_mat;
    float *mom = a.momentum ? a.momentum + mat * a.mom_mat : nullptr;
    constexpr int V = Vec<T>::kLen;
    double squares = 0.0;
    const int vecs = (a.cols + V - 1) / V;
    const int64_t all = int64_t(a.rows) * vecs;
    for (int64_t t = int64_t(blockIdx.x) * kBlock + threadIdx.x; t < all; t += int64_t(gridDim.x) * kBlock) {
        const int64_t r = t / vecs;
        const int i = static_cast<int>(t - r * vecs);
        float g[V];
        load_vec(grad + r * a.grad_row, i, a.cols, g);
        if (mom) {
            float *mr = mom + r * a.mom_row;
#pragma unroll
            for (int h = 0; h < V / 4; ++h) {
                if ((i * (V / 4) + h) * 4 >= a.cols) continue;
                float m[4];
                load_vec(mr, i * (V / 4) + h, a.cols, m);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[j] = a.beta * m[j] + g[4 * h + j];
                    g[4 * h + j] = update_of(a, g[4 * h + j], m[j]);
                }
                store_vec(mr, i * (V / 4) + h, a.cols, m);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (i * V + j < a.cols) squares += static_cast<double>(g[j]) * static_cast<double>(g[j]);
    }
    for (int off = 32; off > 0; off >>= 1) squares += __shfl_xor(squares, off, kWave);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = squares;
    __syncthreads();
    if (threadIdx.x == 0) a.parts[int64_t(mat) * gridDim.x + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

constexpr int kSplitTile = 64;

// X = U / (|U| + eps) times 2^exp in two terms, as U lies (`same`, rows of pad_cols values) and transposed (`turned`, rows of pad_rows values).
// Tiles of 64 x 64 of the padded matrix, zeros past U's own.
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_orth_split(UpdateArgs a, int num_parts, float unit, F16 *__restrict__ same, F16 *__restrict__ turned, int pad_rows, int pad_cols) {
    __shared__ float tile[kSplitTile][kSplitTile + 1];
    __shared__ double lds[kWavesPerBlock];
    const int mat = static_cast<int>(blockIdx.z);
    double squares = 0.0;
    for (int p = static_cast<int>(threadIdx.x); p < num_parts; p += kBlock) squares += a.parts[int64_t(mat) * num_parts + p];
    for (int off = 32; off > 0; off >>= 1) squares += __shfl_xor(squares, off, kWave);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = squares;
    __syncthreads();
    const double norm = sqrt((lds[0] + lds[1]) + (lds[2] + lds[3]));
    const double inv = static_cast<double>(unit) / (norm + static_cast<double>(a.eps));
    const int r0 = static_cast<int>(blockIdx.y) * kSplitTile, c0 = static_cast<int>(blockIdx.x) * kSplitTile;
    const T *grad = static_cast<const T *>(a.grad) + mat * a.grad_mat;
    const float *mom = a.momentum ? a.momentum + mat * a.mom_mat : nullptr;
    const int c = static_cast<int>(threadIdx.x) % kSplitTile;
    for (int r = static_cast<int>(threadIdx.x) / kSplitTile; r < kSplitTile; r += kBlock / kSplitTile) {
        float v = 0.f;
        if (r0 + r < a.rows && c0 + c < a.cols) {
            const float g = static_cast<float>(grad[int64_t(r0 + r) * a.grad_row + c0 + c]);
            v = static_cast<float>(update_of(a, g, mom ? mom[int64_t(r0 + r) * a.mom_row + c0 + c] : 0.f) * inv);
        }
        tile[r][c] = v;
    }
    __syncthreads();
    const int64_t mat_len = int64_t(pad_rows) * pad_cols * 2;
    for (int side = 0; side < 2; ++side) {
        F16 *base = (side ? turned : same) + mat * mat_len;
        const int row0 = side ? c0 : r0, val0 = side ? r0 : c0, len = side ? pad_rows : pad_cols;
        const int row = static_cast<int>(threadIdx.x) / 4, part = static_cast<int>(threadIdx.x) % 4 * 16;      // 16 values of a row
        F16 *to = base + (row0 + row) * (int64_t(len) * 2) + term_at(val0 + part);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Half8 hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                F16 x, y;
                split(side ? tile[part + 8 * h + j][row] : tile[row][part + 8 * h + j], &x, &y);
                hi[j] = x;
                lo[j] = y;
            }
            *reinterpret_cast<Half8 *>(to + 8 * h) = hi;
            *reinterpret_cast<Half8 *>(to + kLineVals + 8 * h) = lo;
        }
    }
}

// ---------------------------------------------------------------- products

enum Epilogue { kGram, kPoly, kIterate, kOut };

struct ProductArgs {
    const F16 *p, *q;                 // P [m x depth], Q [n x depth], in lines
    const F16 *own;                   // [m x n] what the epilogue adds `own_by` times
    F16 *to, *to_turned;              // [m x n], [n x m]
    int64_t p_mat, q_mat, own_mat, to_mat, turned_mat;     // f16 from a matrix of the stack to the next
    int32_t depth;                    // values of a row, a multiple of kLineVals
    int32_t m, n;                     // padded, multiples of the tile
    int32_t tiles_m, tiles_n;
    float acc_by, own_by;
    // the last product
    void *out;                        // update wanted: [m x n] of out_type; or the weights
    int64_t out_row, out_mat;
    int32_t out_m, out_n;             // unpadded
    int32_t out_type;                 // mqg_dtype
    int32_t step;                     // the weights' step: out = keep * out + X
    float keep;
};

// out = acc_by (P Q^T) + own_by own, tiles of (WM FM 32) x (WN FN 32) by WM x WN wavefronts.
template <int EPI, int WM, int WN, int FM, int FN>
__global__ void __launch_bounds__(WM * WN * kWave)
k_orth_product(ProductArgs a) {
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32, kWaves = WM * WN;
    constexpr int kStage = (BM + BN) * kLine;
    __shared__ F16 lds[2 * kStage];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int mat = static_cast<int>(blockIdx.y);
    int tm, tn;
    if constexpr (EPI == kGram || EPI == kPoly) {          // symmetric: the tiles on and below the diagonal
        const int t = static_cast<int>(blockIdx.x);
        tm = static_cast<int>((sqrtf(8.f * static_cast<float>(t) + 1.f) - 1.f) * 0.5f);
        while (tm * (tm + 1) / 2 > t) --tm;
        while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
        tn = t - tm * (tm + 1) / 2;
    } else {
        tm = static_cast<int>(blockIdx.x) / a.tiles_n;
        tn = static_cast<int>(blockIdx.x) - tm * a.tiles_n;
    }
    const int64_t row_len = int64_t(a.depth) * 2;
    const F16 *p = a.p + mat * a.p_mat + int64_t(tm) * BM * row_len;
    const F16 *q = a.q + mat * a.q_mat + int64_t(tn) * BN * row_len;

    // one line of each of the tile's rows: eight rows per instruction of a wavefront, lane l has place l % 8 of row l / 8
    auto fetch = [&](int line, int stage) __attribute__((always_inline)) {
        F16 *to = lds + stage * kStage;
#pragma unroll
        for (int r = 0; r < (BM + BN) / 8; r += kWaves) {
            const int row = (r + wave) * 8 + (lane >> 3);
            const int chunk = chunk_place(row, lane & 7);  // (an exclusive or: its own inverse)
            const F16 *from = (row < BM ? p + row * row_len : q + (row - BM) * row_len) + int64_t(line) * kLine + chunk * 8;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(to + (r + wave) * 8 * kLine), 16, 0, 0);
        }
    };
    Float16v acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Float16v{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    const int wm = wave / WN * FM * 32, wn = wave % WN * FN * 32;
    const int lines = a.depth / kLineVals;
    fetch(0, 0);
    for (int line = 0; line < lines; ++line) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the line has arrived,
        __syncthreads();                                   // in every wavefront, and the other stage has been read
        if (line + 1 < lines) fetch(line + 1, (line + 1) & 1);
        const F16 *at = lds + (line & 1) * kStage;
#pragma unroll
        for (int t = 0; t < 2; ++t) {                      // 16 values at a time
            Half8 ph[FM], pl[FM], qh[FN], ql[FN];
            auto read = [&](int row, int chunk) __attribute__((always_inline)) {
                return *reinterpret_cast<const Half8 *>(at + row * kLine + chunk_place(row, chunk) * 8);
            };
            const int c = 2 * t + (lane >> 5);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int row = wm + i * 32 + (lane & 31);
                ph[i] = read(row, c);
                pl[i] = read(row, c + 4);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int row = BM + wn + j * 32 + (lane & 31);
                qh[j] = read(row, c);
                ql[j] = read(row, c + 4);
            }
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], ql[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[i], qh[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], qh[j], acc[i][j], 0, 0, 0);
                }
        }
    }

    // register e of lane l: row 8 (e / 4) + 4 (l / 32) + e % 4, column l % 32
    const F16 *own = EPI == kGram ? nullptr : a.own + mat * a.own_mat;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int row = tm * BM + wm + i * 32 + 8 * e4 + 4 * (lane >> 5);      // of four
                const int col = tn * BN + wn + j * 32 + (lane & 31);
                float v[4];
                Half4 hi4, lo4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = acc[i][j][4 * e4 + e] * a.acc_by;
                    if constexpr (EPI != kGram) {
                        const F16 *o = own + (row + e) * (int64_t(a.n) * 2) + term_at(col);
                        v[e] += a.own_by * (static_cast<float>(o[0]) + static_cast<float>(o[kLineVals]));
                    }
                    F16 hi, lo;
                    split(v[e], &hi, &lo);
                    hi4[e] = hi;
                    lo4[e] = lo;
                }
                if constexpr (EPI == kOut) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (row + e >= a.out_m || col >= a.out_n) continue;
                        const int64_t at = mat * a.out_mat + (row + e) * a.out_row + col;
                        if (a.step) {
                            float *w = static_cast<float *>(a.out) + at;
                            *w = a.keep * *w + v[e];
                        } else if (a.out_type == MQG_F16) {
                            static_cast<F16 *>(a.out)[at] = static_cast<F16>(v[e]);
                        } else if (a.out_type == MQG_BF16) {
                            static_cast<BF16 *>(a.out)[at] = static_cast<BF16>(v[e]);
                        } else {
                            static_cast<float *>(a.out)[at] = v[e];
                        }
                    }
                } else {
                    F16 *to = a.to + mat * a.to_mat + row * (int64_t(a.n) * 2) + term_at(col);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        to[e * (int64_t(a.n) * 2)] = hi4[e];
                        to[e * (int64_t(a.n) * 2) + kLineVals] = lo4[e];
                    }
                    if (EPI == kIterate || tm != tn) {
                        F16 *turned = (EPI == kIterate ? a.to_turned + mat * a.turned_mat : a.to + mat * a.to_mat) + col * (int64_t(a.m) * 2) + term_at(row);
                        *reinterpret_cast<Half4 *>(turned) = hi4;
                        *reinterpret_cast<Half4 *>(turned + kLineVals) = lo4;
                    }
                }
            }
}

// ---------------------------------------------------------------- host side

// the largest |a x + b x^3 + c x^5| for 0 <= x <= r, and the largest |b t + c t^2| for 0 <= t <= r^2
double poly_most(const float *k, double r) {
    const double a = k[0], b = k[1], c = k[2];
    auto p = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
    double most = p(r);
    auto at = [&](double t) {                              // a stationary point at x^2 = t
        if (t > 0 && t < r * r) most = std::max(most, p(std::sqrt(t)));
    };
    if (c != 0) {
        const double d = 9 * b * b - 20 * a * c;
        if (d >= 0) {
            at((-3 * b + std::sqrt(d)) / (10 * c));
            at((-3 * b - std::sqrt(d)) / (10 * c));
        }
    } else if (b != 0) {
        at(-a / (3 * b));
    }
    return most;
}
double gram_poly_most(const float *k, double r) {
    const double b = k[1], c = k[2], t = r * r;
    double most = std::fabs(t * (b + c * t));
    if (c != 0) {
        const double s = -b / (2 * c);
        if (s > 0 && s < t) most = std::max(most, std::fabs(s * (b + c * s)));
    }
    return most;
}
// the power of two that takes values up to `most` to 2^14 .. 2^15, with a margin for the products' rounding
int unit_exp(double most) {
    int e = 0;
    (void)std::frexp(std::max(most, 0x1p-20) * 1.01, &e);
    return 15 - e;
}

constexpr int kOrthTile = 128;
constexpr int kOrthParts = 256;       // workgroups per matrix that share its norm

struct OrthLayout {
    int64_t n, k;                     // padded
    int64_t x, g;                     // f16 of a matrix
    int64_t parts, bytes;
};
OrthLayout orth_layout(int64_t mats, int64_t rows, int64_t cols) {
    OrthLayout l;
    l.n = ceil_div(std::min(rows, cols), kOrthTile) * kOrthTile;
    l.k = ceil_div(std::max(rows, cols), kOrthTile) * kOrthTile;
    l.x = l.n * l.k * 2;
    l.g = l.n * l.n * 2;
    l.parts = ceil_div(mats * kOrthParts * int64_t(sizeof(double)), 256) * 256;
    l.bytes = l.parts + mats * (3 * l.x + 2 * l.g) * int64_t(sizeof(F16));
    return l;
}

template <int EPI>
int launch_product(mqg_ctx *ctx, ProductArgs a, int64_t mats, hipStream_t s) {
    static const char *const names[] = {"k_orth_gram", "k_orth_poly", "k_orth_iterate", "k_orth_out"};
    a.tiles_m = a.m / kOrthTile;
    a.tiles_n = a.n / kOrthTile;
    const int64_t tiles = EPI == kGram || EPI == kPoly ? int64_t(a.tiles_m) * (a.tiles_m + 1) / 2 : int64_t(a.tiles_m) * a.tiles_n;
    const dim3 grid(static_cast<uint32_t>(tiles), static_cast<uint32_t>(mats));
    MQG_LAUNCH(ctx, names[EPI], s, (k_orth_product<EPI, 2, 2, 2, 2><<<grid, 256, 0, s>>>(a)));
    return MQG_OK;
}

}  // namespace

int64_t orth_scratch_bytes(int64_t mats, int64_t rows, int64_t cols) { return mats > 0 && rows > 0 && cols > 0 ? orth_layout(mats, rows, cols).bytes : 0; }

// Whether the polynomials' values stay in what the iterates are stored in
bool orth_coeffs_fit(const float *coeffs, int32_t steps) {
    double r = 1.0;
    for (int i = 0; i < steps; ++i) {
        const float *k = coeffs + 3 * i;
        if (!std::isfinite(k[0]) || !std::isfinite(k[1]) || !std::isfinite(k[2])) return false;
        const double poly = gram_poly_most(k, r);
        r = poly_most(k, r) * 1.001;
        if (!(r <= 256.0) || !(poly <= 65536.0)) return false;
    }
    return true;
}

int run_orthogonalize(mqg_ctx *ctx, const OrthCall &call, hipStream_t s) {
    const int64_t mats = call.mats, rows = call.rows, cols = call.cols;
    const OrthLayout l = orth_layout(mats, rows, cols);
    int rc = ensure_layer_scratch(ctx, l.bytes, s, call.who);
    if (rc != MQG_OK) return rc;
    double *parts = reinterpret_cast<double *>(ctx->layer_scratch);
    F16 *x = reinterpret_cast<F16 *>(ctx->layer_scratch + l.parts);          // X: n rows of k values
    F16 *xt[2] = {x + mats * l.x, x + 2 * mats * l.x};                       // its transpose, in turns
    F16 *gram = x + 3 * mats * l.x, *poly = gram + mats * l.g;
    const bool tall = rows > cols;

    UpdateArgs u{call.grad, call.momentum, call.grad_row, call.grad_mat, call.mom_row, call.mom_mat, parts, static_cast<int32_t>(rows),
                 static_cast<int32_t>(cols), call.nesterov, call.beta, call.eps};
    double r = 1.0;
    int ex = unit_exp(r);
    const float unit = std::ldexp(1.f, ex);
    const int64_t pad_rows = tall ? l.k : l.n, pad_cols = tall ? l.n : l.k;
    const dim3 split_grid(static_cast<uint32_t>(pad_cols / kSplitTile), static_cast<uint32_t>(pad_rows / kSplitTile), static_cast<uint32_t>(mats));
    F16 *same = tall ? xt[0] : x, *turned = tall ? x : xt[0];
    auto begin = [&](auto type) -> int {
        using T = decltype(type);
        const int64_t vecs = rows * ceil_div(cols, Vec<T>::kLen);
        const int nparts = static_cast<int>(std::min<int64_t>(ceil_div(vecs, kBlock), kOrthParts));
        MQG_LAUNCH(ctx, "k_muon_momentum", s,
                   (k_muon_momentum<T><<<dim3(static_cast<uint32_t>(nparts), static_cast<uint32_t>(mats)), kBlock, 0, s>>>(u)));
        MQG_LAUNCH(ctx, "k_orth_split", s,
                   (k_orth_split<T><<<split_grid, kBlock, 0, s>>>(u, nparts, unit, same, turned, static_cast<int>(pad_rows), static_cast<int>(pad_cols))));
        return MQG_OK;
    };
    rc = call.dtype == MQG_F16 ? begin(F16()) : call.dtype == MQG_BF16 ? begin(BF16()) : begin(float());
    if (rc != MQG_OK) return rc;

    for (int i = 0; i < call.steps; ++i) {
        const float *k = call.coeffs + 3 * i;
        const int eg = unit_exp(r * r), eb = unit_exp(gram_poly_most(k, r));
        ProductArgs a{};
        a.p = a.q = x;
        a.p_mat = a.q_mat = l.x;
        a.depth = static_cast<int32_t>(l.k);
        a.m = a.n = static_cast<int32_t>(l.n);
        a.to = gram;
        a.to_mat = l.g;
        a.acc_by = std::ldexp(1.f, eg - 2 * ex);
        rc = launch_product<kGram>(ctx, a, mats, s);
        if (rc != MQG_OK) return rc;

        a.p = a.q = a.own = gram;
        a.p_mat = a.q_mat = a.own_mat = l.g;
        a.depth = static_cast<int32_t>(l.n);
        a.to = poly;
        a.acc_by = k[2] * std::ldexp(1.f, eb - 2 * eg);
        a.own_by = k[1] * std::ldexp(1.f, eb - eg);
        rc = launch_product<kPoly>(ctx, a, mats, s);
        if (rc != MQG_OK) return rc;

        r = poly_most(k, r) * 1.001;
        const bool last = i + 1 == call.steps;
        const int next = last ? 0 : unit_exp(r);
        F16 *const now = xt[i & 1], *const then = xt[~i & 1];
        const float by = last ? call.out_by : 1.f;
        a.acc_by = by * std::ldexp(1.f, next - eb - ex);
        a.own_by = by * k[0] * std::ldexp(1.f, next - ex);
        // B X as it lies, or, for a tall U, its transpose X^T B: rows of the product are rows of U, so that the output is written along its rows
        a.p = tall ? now : poly;
        a.p_mat = tall ? l.x : l.g;
        a.q = tall ? poly : now;
        a.q_mat = tall ? l.g : l.x;
        a.own = tall ? now : x;
        a.own_mat = a.to_mat = a.turned_mat = l.x;
        a.to = tall ? then : x;
        a.to_turned = tall ? x : then;
        a.m = static_cast<int32_t>(tall ? l.k : l.n);
        a.n = static_cast<int32_t>(tall ? l.n : l.k);
        if (!last) {
            rc = launch_product<kIterate>(ctx, a, mats, s);
        } else {
            a.out = call.out;
            a.out_row = call.out_row;
            a.out_mat = call.out_mat;
            a.out_m = static_cast<int32_t>(rows);
            a.out_n = static_cast<int32_t>(cols);
            a.out_type = call.out_type;
            a.step = call.step;
            a.keep = call.keep;
            rc = launch_product<kOut>(ctx, a, mats, s);
        }
        if (rc != MQG_OK) return rc;
        ex = next;
    }
    return MQG_OK;
}

}  // namespace mqg
