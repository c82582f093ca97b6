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
// Blocks.  A matrix is stored as blocks of 32 rows by 32 values, 4 KB, in the order in which the matrix instruction takes them: the high
// terms' four chunks of eight values, 32 rows each, then the low terms'.  Whatever reads an operand reads 1 KB that lies
// together, from memory to LDS without registers between, from LDS without bank conflicts, or from memory to registers.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "layer_types.h"

namespace mqg {

namespace {

typedef F16 Half8 __attribute__((ext_vector_type(8)));
typedef F16 Half4 __attribute__((ext_vector_type(4)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef float Float16v __attribute__((ext_vector_type(16)));

constexpr int kSide = 32;             // rows and values of a block
constexpr int kBlockLen = 2 * kSide * kSide;     // f16 of a block
constexpr int kTermLen = kSide * kSide;

// Chunk c (values 8 c to 8 c + 7) of row r of a block: its high terms'; the low ones are kTermLen further
__device__ __forceinline__ int chunk_at(int r, int c) { return (c * kSide + r) * 8; }

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
    const uint32_t vecs = static_cast<uint32_t>(a.cols + V - 1) / V, all = static_cast<uint32_t>(a.rows) * vecs;       // 2^30 at most
    for (uint32_t t = blockIdx.x * kBlock + threadIdx.x; t < all; t += gridDim.x * kBlock) {
        const int64_t r = t / vecs;
        const int i = static_cast<int>(t - static_cast<uint32_t>(r) * vecs);
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

// unit / (|U| + eps); 0 for a matrix of zeros without an epsilon, so that zeros stay zeros
__device__ __forceinline__ double unit_over(float unit, double norm, float eps) {
    const double by = norm + static_cast<double>(eps);
    return by == 0.0 ? 0.0 : static_cast<double>(unit) / by;
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
    const int r0 = static_cast<int>(blockIdx.y) * kSplitTile, c0 = static_cast<int>(blockIdx.x) * kSplitTile;
    const T *grad = static_cast<const T *>(a.grad) + mat * a.grad_mat;
    const float *mom = a.momentum ? a.momentum + mat * a.mom_mat : nullptr;
    // the tile's values and the shares of the norm are on their way together
    constexpr int kStep = kBlock / kSplitTile, kEach = kSplitTile / kStep;
    const int c = static_cast<int>(threadIdx.x) % kSplitTile, first = static_cast<int>(threadIdx.x) / kSplitTile;
    const bool col_in = c0 + c < a.cols;
    float v[kEach], m[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int r = r0 + first + k * kStep;
        const bool in = col_in && r < a.rows;
        v[k] = in ? static_cast<float>(grad[int64_t(r) * a.grad_row + c0 + c]) : 0.f;
        m[k] = in && mom ? mom[int64_t(r) * a.mom_row + c0 + c] : 0.f;
    }
    double squares = 0.0;
    for (int p = static_cast<int>(threadIdx.x); p < num_parts; p += kBlock) squares += a.parts[int64_t(mat) * num_parts + p];
    for (int off = 32; off > 0; off >>= 1) squares += __shfl_xor(squares, off, kWave);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = squares;
    __syncthreads();
    const double inv = unit_over(unit, sqrt((lds[0] + lds[1]) + (lds[2] + lds[3])), a.eps);
#pragma unroll
    for (int k = 0; k < kEach; ++k) tile[first + k * kStep][c] = static_cast<float>(update_of(a, v[k], m[k]) * inv);
    __syncthreads();
    const int64_t mat_len = int64_t(pad_rows) * pad_cols * 2;
    for (int side = 0; side < 2; ++side) {                 // 2 x 2 blocks each way, 128 threads to a block
        F16 *base = (side ? turned : same) + mat * mat_len;
        const int row0 = (side ? c0 : r0) / kSide, val0 = (side ? r0 : c0) / kSide, blocks = (side ? pad_rows : pad_cols) / kSide;
        const int row = static_cast<int>(threadIdx.x) % kSide, chunk = static_cast<int>(threadIdx.x) / kSide % 4;
        for (int k = static_cast<int>(threadIdx.x) / 128; k < 4; k += 2) {
            const int rb = k / 2, vb = k % 2;
            Half8 hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = rb * kSide + row, v = vb * kSide + chunk * 8 + j;
                F16 x, y;
                split(side ? tile[v][r] : tile[r][v], &x, &y);
                hi[j] = x;
                lo[j] = y;
            }
            F16 *to = base + (int64_t(row0 + rb) * blocks + val0 + vb) * kBlockLen + chunk_at(row, chunk);
            *reinterpret_cast<Half8 *>(to) = hi;
            *reinterpret_cast<Half8 *>(to + kTermLen) = lo;
        }
    }
}

// ---------------------------------------------------------------- products

enum Epilogue { kGram, kPoly, kIterate, kOut };

struct ProductArgs {
    const F16 *p, *q;                 // P [m x depth], Q [n x depth]
    const F16 *own;                   // [m x n]: what the epilogue adds `own_by` times
    F16 *to, *to_turned;              // [m x n], [n x m]
    int64_t p_mat, q_mat, own_mat, to_mat;     // f16 from a matrix of the stack to the next (to_turned: as to)
    int32_t depth;                    // values of a row
    int32_t m, n;                     // padded, multiples of the tile
    int32_t tiles_m, tiles_n, tiles;  // tiles: of a matrix
    int32_t first_tile;
    float acc_by, own_by;
    // the last product
    void *out;                        // [m x n] of out_type, or the weights
    int64_t out_row, out_mat;
    int32_t out_m, out_n;             // unpadded
    int32_t out_type;                 // mqg_dtype
    int32_t step;                     // the weights' step: out = keep * out + X
    float keep;
};

// Which matrix and tile a workgroup takes.  Workgroups go to the chip's eight dies in turn, each with an L2 of its own: a die gets a run of
// neighbouring tiles, bands of kBand rows of tiles taken column by column, so that the tiles that it works on together share rows and columns.
constexpr int kDies = 8, kBand = 8;
struct TilePlace {
    int mat, m, n;
};
__device__ __forceinline__ int dealt_tile() {
    const int all = static_cast<int>(gridDim.x), id = static_cast<int>(blockIdx.x);
    const int die = id % kDies, more = all % kDies;
    return die * (all / kDies) + (die < more ? die : more) + id / kDies;
}
template <bool SYMMETRIC>
__device__ __forceinline__ TilePlace tile_place(const ProductArgs &a, int at) {
    TilePlace t;
    t.mat = at / a.tiles;
    int i = at - t.mat * a.tiles;
    if constexpr (SYMMETRIC) {                             // the tiles on and below the diagonal: band b has 8 rows of 8 b tiles and a triangle of 36
        int b = static_cast<int>((sqrtf(8.f * static_cast<float>(i) + 1.f) - 1.f) * 0.5f) / kBand;
        while (4 * b * (kBand * b + 1) > i) --b;
        while (4 * (b + 1) * (kBand * (b + 1) + 1) <= i) ++b;
        i -= 4 * b * (kBand * b + 1);
        const int rows = a.tiles_m - b * kBand < kBand ? a.tiles_m - b * kBand : kBand;
        if (i < rows * kBand * b) {
            t.n = i / rows;
            t.m = b * kBand + i - t.n * rows;
        } else {
            i -= rows * kBand * b;
            int r = 0;
            while (i > r) i -= ++r;
            t.m = b * kBand + r;
            t.n = b * kBand + i;
        }
    } else {
        const int b = i / (kBand * a.tiles_n);
        i -= b * kBand * a.tiles_n;
        const int rows = a.tiles_m - b * kBand < kBand ? a.tiles_m - b * kBand : kBand;
        t.n = i / rows;
        t.m = b * kBand + i - t.n * rows;
    }
    return t;
}
static_assert(kBand == 8, "the counts of tiles before a band are written out");

// The epilogue of one block of the product, 32 x 32, whose sums lie in LDS as the matrix instruction leaves them, register e of lane l at
// e * kAccRow + l: row 8 (e / 4) + 4 (l / 32) + e % 4, column l % 32.  PARTS of them, part_len apart, are added; the finished values go back to the
// first, from which they are stored turned.  THREADS threads, t among them, have 128 chunks of eight columns of a row; sync() orders LDS between them.
constexpr int kAccRow = kWave + 4;    // (16 rows of a column in other banks)
constexpr int kAccLen = 16 * kAccRow;
template <int EPI>
__device__ __forceinline__ int unit_row(int u) { return EPI == kOut ? u >> 2 : u % kSide; }        // the output is written along its rows, four threads to each
template <int EPI>
__device__ __forceinline__ int unit_chunk(int u) { return EPI == kOut ? u & 3 : u / kSide; }

// What the epilogue adds, on its way before the sums are there
template <int THREADS>
struct Own {
    static constexpr int kEach = THREADS < 128 ? 128 / THREADS : 1;
    Half8 hi[kEach], lo[kEach];
};
template <int EPI, int THREADS>
__device__ __forceinline__ Own<THREADS> load_own(const ProductArgs &a, int mat, int mb, int nb, int t) {
    Own<THREADS> own;
    if constexpr (EPI != kGram) {
#pragma unroll
        for (int k = 0; k < own.kEach; ++k) {
            const int u = t + k * THREADS < 128 ? t + k * THREADS : 0;
            const F16 *from = a.own + mat * a.own_mat + (int64_t(mb) * (a.n / kSide) + nb) * kBlockLen + chunk_at(unit_row<EPI>(u), unit_chunk<EPI>(u));
            own.hi[k] = *reinterpret_cast<const Half8 *>(from);
            own.lo[k] = *reinterpret_cast<const Half8 *>(from + kTermLen);
        }
    }
    return own;
}

template <int EPI, int PARTS, int THREADS, typename Sync>
__device__ __forceinline__ void finish_block(const ProductArgs &a, const Own<THREADS> &own, float *acc, int part_len, int mat, int mb, int nb, bool mirror, int t,
                                             Sync sync) {
    constexpr int N = Own<THREADS>::kEach;
    auto store = [&](const float (&v)[8], F16 *to) __attribute__((always_inline)) {
        Half8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            F16 x, y;
            split(v[j], &x, &y);
            hi[j] = x;
            lo[j] = y;
        }
        *reinterpret_cast<Half8 *>(to) = hi;
        *reinterpret_cast<Half8 *>(to + kTermLen) = lo;
    };
    const bool mine = THREADS <= 128 || t < 128;
    float v[N][8];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (!mine) break;
        const int u = t + k * THREADS, r = unit_row<EPI>(u), c = unit_chunk<EPI>(u);
        float *at = acc + ((r >> 3) * 4 + (r & 3)) * kAccRow + 32 * ((r >> 2) & 1) + 8 * c;
        Float4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            x += *reinterpret_cast<const Float4 *>(at + p * part_len);
            y += *reinterpret_cast<const Float4 *>(at + p * part_len + 4);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[k][j] = (j < 4 ? x[j % 4] : y[j % 4]) * a.acc_by;
            // (as one operation: the compiler would choose which product to round, and not in all kernels the same)
            if constexpr (EPI != kGram) v[k][j] = fmaf(a.own_by, static_cast<float>(own.hi[k][j]) + static_cast<float>(own.lo[k][j]), v[k][j]);
        }
        if (EPI == kIterate || (EPI != kOut && mirror)) {
            *reinterpret_cast<Float4 *>(at) = Float4{v[k][0], v[k][1], v[k][2], v[k][3]};
            *reinterpret_cast<Float4 *>(at + 4) = Float4{v[k][4], v[k][5], v[k][6], v[k][7]};
        }
    }
    if constexpr (EPI == kOut) {
        if (a.step) {                                      // all weights are on their way before the first is written
            float w[N][2][4];
            auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int u = t + k * THREADS, row = mb * kSide + unit_row<EPI>(u), col0 = nb * kSide + 8 * unit_chunk<EPI>(u);
                    if (!mine || row >= a.out_m) continue;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (col0 + 4 * h < a.out_n) f(static_cast<float *>(a.out) + mat * a.out_mat + row * a.out_row, col0 / 4 + h, k, h);
                }
            };
            each([&](const float *at, int i, int k, int h) __attribute__((always_inline)) { load_vec(at, i, a.out_n, w[k][h]); });
            each([&](float *at, int i, int k, int h) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) w[k][h][j] = fmaf(a.keep, w[k][h][j], v[k][4 * h + j]);
                store_vec(at, i, a.out_n, w[k][h]);
            });
            return;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int u = t + k * THREADS, row = mb * kSide + unit_row<EPI>(u), col0 = nb * kSide + 8 * unit_chunk<EPI>(u);
            if (!mine || row >= a.out_m) continue;
            const int64_t to = mat * a.out_mat + row * a.out_row;
            if (a.out_type == MQG_F16) {
                store_vec(static_cast<F16 *>(a.out) + to, col0 / 8, a.out_n, v[k]);
            } else if (a.out_type == MQG_BF16) {
                store_vec(static_cast<BF16 *>(a.out) + to, col0 / 8, a.out_n, v[k]);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float z[4] = {v[k][4 * h], v[k][4 * h + 1], v[k][4 * h + 2], v[k][4 * h + 3]};
                    store_vec(static_cast<float *>(a.out) + to, col0 / 4 + h, a.out_n, z);
                }
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int u = t + k * THREADS;
            if (mine) store(v[k], a.to + mat * a.to_mat + (int64_t(mb) * (a.n / kSide) + nb) * kBlockLen + chunk_at(unit_row<EPI>(u), unit_chunk<EPI>(u)));
        }
        if (EPI != kIterate && !mirror) return;            // (the same in all threads of a tile)
        sync();
#pragma unroll
        for (int k = 0; k < N; ++k) {                      // eight rows of a column
            const int u = t + k * THREADS, col = u % kSide, c = u / kSide;
            if (!mine) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = acc[(c * 4 + (j & 3)) * kAccRow + col + 32 * (j >> 2)];
            store(v[k], a.to_turned + mat * a.to_mat + (int64_t(nb) * (a.m / kSide) + mb) * kBlockLen + chunk_at(col, c));
        }
    }
}

// out = acc_by (P Q^T) + own_by own, tiles of (WM FM 32) x (WN FN 32) by WM x WN wavefronts, blocks through LDS, the
// next ones on their way while these are multiplied.
template <int EPI, int WM, int WN, int FM, int FN>
__global__ void __launch_bounds__(WM * WN * kWave)
k_orth_product(ProductArgs a) {
    constexpr int BM = WM * FM, BN = WN * FN, kWaves = WM * WN;            // the tile in blocks
    constexpr int kStage = (BM + BN) * kBlockLen, kLoads = (BM + BN) * 4 / kWaves;      // of a wavefront
    static_assert(kWaves * kAccLen * sizeof(float) <= 2 * kStage * sizeof(F16), "the epilogue's blocks fit");
    __shared__ __attribute__((aligned(16))) F16 lds[2 * kStage];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const TilePlace tile = tile_place<EPI == kGram || EPI == kPoly>(a, dealt_tile());
    const int deep = a.depth / kSide;
    const F16 *p = a.p + tile.mat * a.p_mat + int64_t(tile.m) * BM * deep * kBlockLen;
    const F16 *q = a.q + tile.mat * a.q_mat + int64_t(tile.n) * BN * deep * kBlockLen;

    // blocks number `line` of the tile's rows of blocks, 1 KB an instruction of a wavefront
    auto fetch = [&](int line, int stage) __attribute__((always_inline)) {
        F16 *to = lds + stage * kStage;
        const int64_t at = int64_t(line) * kBlockLen + lane * 8;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int unit = u * kWaves + wave, b = unit / 4;
            const F16 *from = (b < BM ? p + int64_t(b) * deep * kBlockLen : q + int64_t(b - BM) * deep * kBlockLen) + (unit % 4) * 512 + at;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(to + unit * 512), 16, 0, 0);
        }
    };
    Float16v acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Float16v{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    const int wm = wave / WN * FM, wn = wave % WN * FN;
    struct Operands {                 // of 16 values
        Half8 ph[FM], pl[FM], qh[FN], ql[FN];
    };
    auto read = [&](int stage, int t) __attribute__((always_inline)) {
        const F16 *at = lds + stage * kStage + t * 512 + lane * 8;
        Operands o;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            o.ph[i] = *reinterpret_cast<const Half8 *>(at + (wm + i) * kBlockLen);
            o.pl[i] = *reinterpret_cast<const Half8 *>(at + (wm + i) * kBlockLen + kTermLen);
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            o.qh[j] = *reinterpret_cast<const Half8 *>(at + (BM + wn + j) * kBlockLen);
            o.ql[j] = *reinterpret_cast<const Half8 *>(at + (BM + wn + j) * kBlockLen + kTermLen);
        }
        return o;
    };
    auto multiply = [&](const Operands &o) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.ph[i], o.ql[j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.pl[i], o.qh[j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.ph[i], o.qh[j], acc[i][j], 0, 0, 0);
            }
    };
    constexpr int kReads = 2 * (FM + FN), kProducts = 3 * FM * FN;
    fetch(0, 0);
    for (int line = 0; line < deep; ++line) {
        // the line has arrived and this wavefront's reads of the other stage are done; behind the barrier that holds for all
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (line + 1 < deep) fetch(line + 1, (line + 1) & 1);
        const Operands first = read(line & 1, 0), second = read(line & 1, 1);
        multiply(first);
        multiply(second);
        // the second half's reads between the first half's products, one and one
        __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
        for (int k = 0; k < kReads; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 2 * kProducts - kReads, 0);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");     // the stages are free
    float *mine = reinterpret_cast<float *>(lds) + wave * kAccLen;
    const int mb = tile.m * BM + wm, nb = tile.n * BN + wn;
    Own<kWave> next = load_own<EPI, kWave>(a, tile.mat, mb, nb, lane);
#pragma unroll
    for (int b = 0; b < FM * FN; ++b) {
        const int i = b / FN, j = b % FN;
        const Own<kWave> own = next;
        if (b + 1 < FM * FN) next = load_own<EPI, kWave>(a, tile.mat, mb + (b + 1) / FN, nb + (b + 1) % FN, lane);
#pragma unroll
        for (int e = 0; e < 16; ++e) mine[e * kAccRow + lane] = acc[i][j][e];
        wave_lds_sync();
        finish_block<EPI, 1, kWave>(a, own, mine, 0, tile.mat, mb + i, nb + j, tile.m != tile.n, lane, [] { wave_lds_sync(); });
        wave_lds_sync();
    }
}

// The same for few tiles: F x F blocks of the product to a workgroup, whose depth eight wavefronts share.  Each takes every eighth block of P
// and of Q, from memory to registers, AHEAD of them on their way together, and their sums are added in LDS.  (Sixteen: no faster.)
// SUB > 1: the blocks of the tiles of SUB x SUB blocks from number first_tile on.
constexpr int kFewWaves = 8;
template <int EPI, int SUB, int F, int AHEAD>
__global__ void __launch_bounds__(kFewWaves * kWave) __attribute__((amdgpu_waves_per_eu(F == 1 ? 4 : 2, F == 1 ? 4 : 2)))
k_orth_product_few(ProductArgs a) {
    constexpr bool symmetric = EPI == kGram || EPI == kPoly;
    static_assert(SUB == 1 || F == 1, "");
    __shared__ __attribute__((aligned(16))) float lds[kFewWaves * F * F * kAccLen];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    TilePlace tile = tile_place<symmetric>(a, SUB == 1 ? dealt_tile() : a.first_tile + static_cast<int>(blockIdx.x) / (SUB * SUB));
    const bool mirror = tile.m != tile.n;
    if constexpr (SUB > 1) {
        const int sub = static_cast<int>(blockIdx.x) % (SUB * SUB);
        tile.m = tile.m * SUB + sub / SUB;
        tile.n = tile.n * SUB + sub % SUB;
    }
    const int deep = a.depth / kSide;
    const F16 *p = a.p + tile.mat * a.p_mat + int64_t(tile.m) * F * deep * kBlockLen + lane * 8;
    const F16 *q = a.q + tile.mat * a.q_mat + int64_t(tile.n) * F * deep * kBlockLen + lane * 8;
    Float16v acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = Float16v{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    // N blocks from number `line` on: all their loads, then their products
    auto batch = [&](int line, auto number) __attribute__((always_inline)) {
        constexpr int N = decltype(number)::value;
        Half8 pv[N][F][4], qv[N][F][4];                    // high terms of the block's halves, low terms
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t at = (int64_t(i) * deep + line + u * kFewWaves) * kBlockLen + k * 512;
                    pv[u][i][k] = *reinterpret_cast<const Half8 *>(p + at);
                    qv[u][i][k] = *reinterpret_cast<const Half8 *>(q + at);
                }
        __builtin_amdgcn_sched_barrier(0);                 // (the compiler would put every load where it is used, one after the other)
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pv[u][i][t], qv[u][j][2 + t], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pv[u][i][2 + t], qv[u][j][t], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pv[u][i][t], qv[u][j][t], acc[i][j], 0, 0, 0);
                    }
    };
    using std::integral_constant;
    int line = wave, left = (deep - wave + kFewWaves - 1) / kFewWaves;
    for (; left >= AHEAD; left -= AHEAD, line += AHEAD * kFewWaves) batch(line, integral_constant<int, AHEAD>());
    if (AHEAD > 2 && left == 2) batch(line, integral_constant<int, 2>());
    if (left == 1) batch(line, integral_constant<int, 1>());
    constexpr int kThreads = kFewWaves * kWave / (F * F);  // to a block
    const int b = static_cast<int>(threadIdx.x) / kThreads, mb = tile.m * F + b / F, nb = tile.n * F + b % F;
    const Own<kThreads> own = load_own<EPI, kThreads>(a, tile.mat, mb, nb, static_cast<int>(threadIdx.x) % kThreads);
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) lds[(wave * F * F + i * F + j) * kAccLen + e * kAccRow + lane] = acc[i][j][e];
    __syncthreads();
    finish_block<EPI, kFewWaves, kThreads>(a, own, lds + b * kAccLen, F * F * kAccLen, tile.mat, mb, nb, mirror, static_cast<int>(threadIdx.x) % kThreads,
                                           [] { __syncthreads(); });
}

// ---------------------------------------------------------------- small matrices

// What the matrix instruction leaves in a lane are four times four neighbouring values of a column: half of chunk c of row lane % 32 of the block turned.
__device__ __forceinline__ int turned_at(int lane, int c) { return chunk_at(lane & 31, c) + 4 * (lane >> 5); }
__device__ __forceinline__ void store_turned(F16 *block, int lane, const Float16v &v) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        Half4 hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            F16 h, l;
            split(v[4 * c + j], &h, &l);
            hi[j] = h;
            lo[j] = l;
        }
        F16 *to = block + turned_at(lane, c);
        *reinterpret_cast<Half4 *>(to) = hi;
        *reinterpret_cast<Half4 *>(to + kTermLen) = lo;
    }
}
// v <- by v + own_by (the block turned)
__device__ __forceinline__ void add_turned(Float16v &v, float by, const F16 *block, int lane, float own_by) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const F16 *own = block + turned_at(lane, c);
        const Half4 hi = *reinterpret_cast<const Half4 *>(own), lo = *reinterpret_cast<const Half4 *>(own + kTermLen);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * c + j] = fmaf(own_by, static_cast<float>(hi[j]) + static_cast<float>(lo[j]), by * v[4 * c + j]);
    }
}

// What the three products of a step multiply their sums and their own values by
struct StepScales {
    float gram, poly, poly_own, x, x_own;
};

struct SmallArgs {
    UpdateArgs u;
    float unit;                       // of the first X
    int32_t steps;
    StepScales by[MQG_ORTH_MAX_STEPS];
    void *out;
    int64_t out_row, out_mat;
    int32_t out_type, step;
    float keep;
};

// Word k of lane q of every four lanes becomes word q of lane k.
__device__ __forceinline__ void quad_transpose(uint32_t (&w)[4]) {
    const bool odd = lane_id() & 1, upper = lane_id() & 2;
#pragma unroll
    for (int k = 0; k < 4; k += 2) {                       // with the neighbour: words 0 and 1, 2 and 3
        const uint32_t out = odd ? w[k] : w[k + 1], in = dpp_u32<0xB1>(out);
        if (odd) w[k] = in;
        else w[k + 1] = in;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {                          // with the lane two further: words 0 and 2, 1 and 3
        const uint32_t out = upper ? w[k] : w[k + 2], in = dpp_u32<0x4E>(out);
        if (upper) w[k] = in;
        else w[k + 2] = in;
    }
}

// A matrix whose X, X^T and G (then B) fit a compute unit's LDS, all of it in one launch: a workgroup holds it from the update to the
// weights.  What bounds it is latency: three products of a few blocks per step, with the LDS written between two barriers: 16 x 16 15.5 us, 64 x 64 20.5, 64 x 256 39.3 for
// five steps (by the kernels below 57, 70 and 70).
constexpr int kSmallWaves = 8, kSmallBlocks = 39, kSmallMost = 16;      // blocks of LDS; of X
inline bool orth_fits_small(int64_t n, int64_t k) {
    const int64_t nb = ceil_div(n, kSide), kb = ceil_div(k, kSide);
    return nb * kb <= kSmallMost && 2 * nb * kb + nb * nb <= kSmallBlocks;
}
template <typename T>
__global__ void __launch_bounds__(kSmallWaves * kWave)
k_orth_small(SmallArgs a) {
    constexpr int kThreads = kSmallWaves * kWave, kGramEach = 2, kIterateEach = kSmallMost / kSmallWaves;
    __shared__ __attribute__((aligned(16))) F16 lds[kSmallBlocks * kBlockLen];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)), tid = static_cast<int>(threadIdx.x);
    const int mat = static_cast<int>(blockIdx.x);
    const int rows = a.u.rows, cols = a.u.cols;
    const bool tall = rows > cols;
    const int nb = ((tall ? cols : rows) + kSide - 1) / kSide, kb = ((tall ? rows : cols) + kSide - 1) / kSide;
    F16 *x = lds, *xt = lds + nb * kb * kBlockLen, *gram = xt + nb * kb * kBlockLen;
    // the update, row by row of X with a few values between the rows, where X^T will be (and the first KB of G)
    float *raw = reinterpret_cast<float *>(xt);
    double *norms = reinterpret_cast<double *>(gram + nb * nb * kBlockLen) - kSmallWaves;
    const int raw_row = kb * kSide + 4;
    if (rows * cols < nb * kb * kSide * kSide) {
        for (int i = tid; i < nb * kSide * raw_row; i += kThreads) raw[i] = 0.f;
        __syncthreads();
    }
    const T *grad = static_cast<const T *>(a.u.grad) + mat * a.u.grad_mat;
    float *mom = a.u.momentum ? a.u.momentum + mat * a.u.mom_mat : nullptr;
    double squares = 0.0;
    constexpr int V = 4, kAhead = 4;                       // vectors of a row on their way together
    const int vecs = (cols + V - 1) / V, all = rows * vecs;
    auto four = [&](const auto *row, int i, float (&v)[V]) __attribute__((always_inline)) {
        using E = std::remove_cv_t<std::remove_pointer_t<decltype(row)>>;
        typedef E Four __attribute__((ext_vector_type(4)));
        typedef Four AnyFour __attribute__((aligned(sizeof(E))));
        if ((i + 1) * V <= cols) {
            const Four x4 = *reinterpret_cast<const AnyFour *>(row + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = static_cast<float>(x4[j]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = i * V + j < cols ? static_cast<float>(row[i * V + j]) : 0.f;
        }
    };
    for (int i0 = tid; i0 < all; i0 += kAhead * kThreads) {
        float g[kAhead][V], m[kAhead][V];
        int r[kAhead], i[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = i0 + k * kThreads < all ? i0 + k * kThreads : i0;
            r[k] = static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(vecs));
            i[k] = at - r[k] * vecs;
            four(grad + r[k] * a.u.grad_row, i[k], g[k]);
            if (mom) four(mom + r[k] * a.u.mom_row, i[k], m[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k * kThreads >= all) break;
            if (mom) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    m[k][j] = a.u.beta * m[k][j] + g[k][j];
                    g[k][j] = update_of(a.u, g[k][j], m[k][j]);
                }
                store_vec(mom + r[k] * a.u.mom_row, i[k], cols, m[k]);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = i[k] * V + j;
                if (c >= cols) continue;
                squares += static_cast<double>(g[k][j]) * static_cast<double>(g[k][j]);
                raw[tall ? c * raw_row + r[k] : r[k] * raw_row + c] = g[k][j];
            }
        }
    }
    for (int off = 32; off > 0; off >>= 1) squares += __shfl_xor(squares, off, kWave);
    if (lane == 0) norms[wave] = squares;
    __syncthreads();
    squares = 0.0;
#pragma unroll
    for (int k = 0; k < kSmallWaves; ++k) squares += norms[k];
    // unit / (|U| + eps) as a number of 32 bits and a power of two: no product leaves the range of 32 bits on its way
    int exp = 0;
    const float inv = static_cast<float>(frexp(unit_over(a.unit, sqrt(squares), a.u.eps), &exp));
    const int chunks = nb * kb * 128;
    constexpr int kChunksEach = kSmallMost * 128 / kThreads;
    auto store_chunk = [&](F16 *to, Half8 hi, Half8 lo) __attribute__((always_inline)) {
        *reinterpret_cast<Half8 *>(to) = hi;
        *reinterpret_cast<Half8 *>(to + kTermLen) = lo;
    };
    auto chunk_of = [&](const float *from, int step, Half8 *hi, Half8 *lo) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // in this order: a product of numbers below 2^-126 would lose bits; rounded to 32 bits before it is split: the compiler would make one operation of both
            float v = ldexpf(from[j * step], exp) * inv;
            asm("" : "+v"(v));
            F16 h, l;
            split(v, &h, &l);
            (*hi)[j] = h;
            (*lo)[j] = l;
        }
    };
    Half8 hi[kChunksEach], lo[kChunksEach];
#pragma unroll
    for (int e = 0; e < kChunksEach; ++e) {
        const int u = tid + e * kThreads, b = u / 128, r = u % kSide, c = u / kSide % 4;
        if (u >= chunks) break;
        Half8 h, l;
        chunk_of(raw + (b / kb * kSide + r) * raw_row + b % kb * kSide + 8 * c, 1, &h, &l);            // of X: eight values of a row
        store_chunk(x + b * kBlockLen + chunk_at(r, c), h, l);
        chunk_of(raw + (b % nb * kSide + 8 * c) * raw_row + b / nb * kSide + r, raw_row, &hi[e], &lo[e]);      // of X^T: eight rows of a column
    }
    __syncthreads();                                       // X^T in the place of the update
#pragma unroll
    for (int e = 0; e < kChunksEach; ++e) {
        const int u = tid + e * kThreads;
        if (u >= chunks) break;
        store_chunk(xt + u / 128 * kBlockLen + chunk_at(u % kSide, u / kSide % 4), hi[e], lo[e]);
    }
    __syncthreads();

    int own_lane = lane;              // made new in every step: the compiler would keep the addresses of all of a step's accesses, 256 registers and more
    // sum over `deep` neighbouring blocks of P and Q
    auto product = [&](const F16 *p, const F16 *q, int deep) __attribute__((always_inline)) {
        Float16v acc{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        for (int d = 0; d < deep; ++d) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const F16 *pb = p + d * kBlockLen + t * 512 + own_lane * 8, *qb = q + d * kBlockLen + t * 512 + own_lane * 8;
                const Half8 ph = *reinterpret_cast<const Half8 *>(pb), pl = *reinterpret_cast<const Half8 *>(pb + kTermLen);
                const Half8 qh = *reinterpret_cast<const Half8 *>(qb), ql = *reinterpret_cast<const Half8 *>(qb + kTermLen);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
            }
        }
        return acc;
    };
    Float16v v[kIterateEach];
#pragma unroll 1
    for (int s = 0;; ++s) {
        const StepScales by = a.by[s];
        asm volatile("" : "+v"(own_lane));
        for (int b = wave; b < nb * nb; b += kSmallWaves) {                  // G: every block is computed, and stored turned
            const int i = b / nb, j = b % nb;
            Float16v g = product(x + i * kb * kBlockLen, x + j * kb * kBlockLen, kb);
            g *= by.gram;
            store_turned(gram + (j * nb + i) * kBlockLen, own_lane, g);
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kGramEach; ++e) {
            const int b = wave + e * kSmallWaves, i = b / nb, j = b % nb;
            if (b >= nb * nb) continue;
            v[e] = product(gram + i * nb * kBlockLen, gram + j * nb * kBlockLen, nb);
            add_turned(v[e], by.poly, gram + (j * nb + i) * kBlockLen, own_lane, by.poly_own);
        }
        __syncthreads();                                   // B in the place of G
#pragma unroll
        for (int e = 0; e < kGramEach; ++e) {
            const int b = wave + e * kSmallWaves;
            if (b < nb * nb) store_turned(gram + (b % nb * nb + b / nb) * kBlockLen, own_lane, v[e]);
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kIterateEach; ++e) {           // block (i, j) of X
            const int b = wave + e * kSmallWaves, i = b / kb, j = b % kb;
            if (b >= nb * kb) continue;
            v[e] = product(gram + i * nb * kBlockLen, xt + j * nb * kBlockLen, nb);
            add_turned(v[e], by.x, xt + (j * nb + i) * kBlockLen, own_lane, by.x_own);
        }
        if (s + 1 == a.steps) break;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kIterateEach; ++e) {
            const int b = wave + e * kSmallWaves, i = b / kb, j = b % kb;
            if (b >= nb * kb) continue;
            store_turned(xt + (j * nb + i) * kBlockLen, own_lane, v[e]);
            // as it lies: four lanes exchange their four rows of a column each for a row of four columns each
            F16 *block = x + b * kBlockLen + chunk_at(4 * (own_lane >> 5) + (own_lane & 3), (own_lane & 31) / 8) + (own_lane & 4);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    F16 h, l;
                    split(v[e][4 * c + k], &h, &l);
                    w[k] = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, h)) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, l)) << 16;
                }
                quad_transpose(w);
                typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
                F16 *to = block + 8 * 8 * c;
                *reinterpret_cast<Words2 *>(to) = Words2{(w[0] & 0xFFFFu) | w[1] << 16, (w[2] & 0xFFFFu) | w[3] << 16};
                *reinterpret_cast<Words2 *>(to + kTermLen) = Words2{w[0] >> 16 | (w[1] & 0xFFFF0000u), w[2] >> 16 | (w[3] & 0xFFFF0000u)};
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < kIterateEach; ++e) {
        const int b = wave + e * kSmallWaves, i = b / kb, j = b % kb;
        if (b >= nb * kb) continue;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int m = i * kSide + 8 * (k / 4) + 4 * (lane >> 5) + k % 4, n = j * kSide + (lane & 31);
            const int r = tall ? n : m, c = tall ? m : n;
            if (r >= rows || c >= cols) continue;
            const int64_t at = mat * a.out_mat + r * a.out_row + c;
            if (a.step) {
                float *w = static_cast<float *>(a.out) + at;
                *w = fmaf(a.keep, *w, v[e][k]);
            } else if (a.out_type == MQG_F16) {
                static_cast<F16 *>(a.out)[at] = static_cast<F16>(v[e][k]);
            } else if (a.out_type == MQG_BF16) {
                static_cast<BF16 *>(a.out)[at] = static_cast<BF16>(v[e][k]);
            } else {
                static_cast<float *>(a.out)[at] = v[e][k];
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

// Which kernel makes a product, by the tiles of 64 x 64 that it has, both halves of a symmetric one counted.  Times in us by events of single blocks
// (kBlocks), tiles of 64 and of 128:  1,024^2 G 13.7, 13.4, 28, X 17.4, 14.6, 31;  512^2 7.3, 9.6, 19 and 8.3, 10.2, 20;  512 x 4,096 16, 32, 85 and 21, 18, 24;
// two of 1,024^2 18.5, 21.7, 29 and 28, 23, 33;  four 29.5, 30.5, 31.5 and 51, 42, 38;  eight 53, 48, 51 and 99, 80, 63;  1,536^2 25, 28, 39 and 43, 42, 44;  2,048^2 52, 52, 50
// and 91, 71, 62;  4,096^2 366, 268, 218 and 728, 529, 397.  (Tiles of 64 through LDS with two to five blocks ahead: as those of 64 in all of these.)
enum Kernel { kBlocks, kTiles64, kTiles128 };
Kernel kernel_for(bool symmetric, int64_t m, int64_t n, int64_t mats) {
    const int64_t tiles = ceil_div(m, 64) * ceil_div(n, 64) * mats;
    if (tiles <= (symmetric ? 600 : 144)) return kBlocks;
    return tiles <= (symmetric ? 2048 : 768) ? kTiles64 : kTiles128;
}

constexpr int kOrthParts = 1024;      // workgroups per matrix that share its norm

struct OrthLayout {
    int64_t n, k;                     // padded
    int64_t x, g;                     // f16 of a matrix
    int64_t parts, bytes;
    Kernel gram_kernel, x_kernel;
};
OrthLayout orth_layout(int64_t mats, int64_t rows, int64_t cols) {
    OrthLayout l;
    const int64_t n = std::min(rows, cols), k = std::max(rows, cols);
    l.gram_kernel = kernel_for(true, n, n, mats);
    l.x_kernel = kernel_for(false, n, k, mats);
    const int64_t pad = l.gram_kernel == kTiles128 || l.x_kernel == kTiles128 ? 128 : 64;
    l.n = ceil_div(n, pad) * pad;
    l.k = ceil_div(k, pad) * pad;
    l.x = l.n * l.k * 2;
    l.g = l.n * l.n * 2;
    l.parts = ceil_div(mats * kOrthParts * int64_t(sizeof(double)), 256) * 256;
    l.bytes = l.parts + mats * (3 * l.x + 2 * l.g) * int64_t(sizeof(F16));
    return l;
}

// Two tiles of 128 x 128 fit a compute unit.  A few tiles more than whole rounds of the chip would take as long as a round (4,096 rows: 528
// tiles, G of 8,192 values 534 us); up to kTileRest of them go block by block, their depth shared by the wavefronts (387 and 30).
constexpr int kTileRound = 512, kTileRest = 64;
template <int EPI>
int launch_product(mqg_ctx *ctx, ProductArgs a, int64_t mats, Kernel kernel, hipStream_t s) {
    static const char *const names[] = {"k_orth_gram", "k_orth_poly", "k_orth_iterate", "k_orth_out"};
    constexpr bool symmetric = EPI == kGram || EPI == kPoly;
    auto tiles_of = [&](int side) {
        a.tiles_m = a.m / side;
        a.tiles_n = a.n / side;
        a.tiles = symmetric ? static_cast<int32_t>(int64_t(a.tiles_m) * (a.tiles_m + 1) / 2) : a.tiles_m * a.tiles_n;
        return static_cast<int>(a.tiles * mats);
    };
    if (kernel == kBlocks) {
        const int grid = tiles_of(kSide);
        MQG_LAUNCH(ctx, names[EPI], s, (k_orth_product_few<EPI, 1, 1, 3><<<grid, kFewWaves * kWave, 0, s>>>(a)));
        return MQG_OK;
    }
    if (kernel == kTiles64) {
        const int grid = tiles_of(64);
        MQG_LAUNCH(ctx, names[EPI], s, (k_orth_product_few<EPI, 1, 2, 2><<<grid, kFewWaves * kWave, 0, s>>>(a)));
        return MQG_OK;
    }
    if constexpr (!symmetric) {
        // Whole rounds of tiles of 256, one to a compute unit: half the operands' traffic.  8,192 x 4,096: 763 -> 698 us (1,180 TFLOP/s of f16 products; the same
        // without any traffic 572, with the products alone 525: the card's clock falls to 1.5 GHz under them), 4,096^2 390 -> 356; 24 of 1,024^2, a round and a half, 180 and 198.
        if (a.m % 256 == 0 && a.n % 256 == 0) {
            const int64_t wide = tiles_of(256), rounds = ceil_div(wide, 256);
            if (wide * 10 >= rounds * 256 * 9) {
                MQG_LAUNCH(ctx, names[EPI], s, (k_orth_product<EPI, 2, 4, 4, 2><<<static_cast<int>(wide), 512, 0, s>>>(a)));
                return MQG_OK;
            }
        }
    }
    const int all = tiles_of(128), rest = all > kTileRound && all % kTileRound <= kTileRest ? all % kTileRound : 0;
    MQG_LAUNCH(ctx, names[EPI], s, (k_orth_product<EPI, 2, 2, 2, 2><<<all - rest, 256, 0, s>>>(a)));
    if (rest) {
        constexpr int sub = 128 / kSide;
        a.first_tile = all - rest;
        MQG_LAUNCH(ctx, names[EPI], s, (k_orth_product_few<EPI, sub, 1, 3><<<rest * sub * sub, kFewWaves * kWave, 0, s>>>(a)));
    }
    return MQG_OK;
}

}  // namespace

int64_t orth_scratch_bytes(int64_t mats, int64_t rows, int64_t cols) {
    if (mats <= 0 || rows <= 0 || cols <= 0 || orth_fits_small(std::min(rows, cols), std::max(rows, cols))) return 0;
    return orth_layout(mats, rows, cols).bytes;
}

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
    UpdateArgs u{call.grad, call.momentum, call.grad_row, call.grad_mat, call.mom_row, call.mom_mat, nullptr, static_cast<int32_t>(rows),
                 static_cast<int32_t>(cols), call.nesterov, call.beta, call.eps};
    // the powers of two that X, G and B are stored times, step by step
    StepScales by[MQG_ORTH_MAX_STEPS];
    double r = 1.0;
    int ex = unit_exp(r);
    const float unit = std::ldexp(1.f, ex);
    for (int i = 0; i < call.steps; ++i) {
        const float *k = call.coeffs + 3 * i;
        const bool last = i + 1 == call.steps;
        const int eg = unit_exp(r * r), eb = unit_exp(gram_poly_most(k, r));
        r = poly_most(k, r) * 1.001;
        const int next = last ? 0 : unit_exp(r);
        const float out_by = last ? call.out_by : 1.f;
        by[i] = {std::ldexp(1.f, eg - 2 * ex), k[2] * std::ldexp(1.f, eb - 2 * eg), k[1] * std::ldexp(1.f, eb - eg),
                 out_by * std::ldexp(1.f, next - eb - ex), out_by * k[0] * std::ldexp(1.f, next - ex)};
        ex = next;
    }
    auto typed = [&](auto go) { return call.dtype == MQG_F16 ? go(F16()) : call.dtype == MQG_BF16 ? go(BF16()) : go(float()); };

    if (orth_fits_small(std::min(rows, cols), std::max(rows, cols))) {
        SmallArgs a{};
        a.u = u;
        a.unit = unit;
        a.steps = call.steps;
        std::copy(by, by + call.steps, a.by);
        a.out = call.out;
        a.out_row = call.out_row;
        a.out_mat = call.out_mat;
        a.out_type = call.out_type;
        a.step = call.step;
        a.keep = call.keep;
        return typed([&](auto type) -> int {
            using T = decltype(type);
            MQG_LAUNCH(ctx, "k_orth_small", s, (k_orth_small<T><<<static_cast<int>(mats), kSmallWaves * kWave, 0, s>>>(a)));
            return MQG_OK;
        });
    }

    const OrthLayout l = orth_layout(mats, rows, cols);
    int rc = ensure_layer_scratch(ctx, l.bytes, s, call.who);
    if (rc != MQG_OK) return rc;
    u.parts = reinterpret_cast<double *>(ctx->layer_scratch.data);
    F16 *x = reinterpret_cast<F16 *>(ctx->layer_scratch.data + l.parts);          // X: n rows of k values
    F16 *xt[2] = {x + mats * l.x, x + 2 * mats * l.x};                       // its transpose, in turns
    F16 *gram = x + 3 * mats * l.x, *poly = gram + mats * l.g;
    const bool tall = rows > cols;
    const int64_t pad_rows = tall ? l.k : l.n, pad_cols = tall ? l.n : l.k;
    const dim3 split_grid(static_cast<uint32_t>(pad_cols / kSplitTile), static_cast<uint32_t>(pad_rows / kSplitTile), static_cast<uint32_t>(mats));
    F16 *same = tall ? xt[0] : x, *turned = tall ? x : xt[0];
    rc = typed([&](auto type) -> int {
        using T = decltype(type);
        const int64_t vecs = rows * ceil_div(cols, Vec<T>::kLen);
        const int nparts = static_cast<int>(std::min<int64_t>(ceil_div(vecs, kBlock), kOrthParts));
        MQG_LAUNCH(ctx, "k_muon_momentum", s,
                   (k_muon_momentum<T><<<dim3(static_cast<uint32_t>(nparts), static_cast<uint32_t>(mats)), kBlock, 0, s>>>(u)));
        MQG_LAUNCH(ctx, "k_orth_split", s,
                   (k_orth_split<T><<<split_grid, kBlock, 0, s>>>(u, nparts, unit, same, turned, static_cast<int>(pad_rows), static_cast<int>(pad_cols))));
        return MQG_OK;
    });
    if (rc != MQG_OK) return rc;

    for (int i = 0; i < call.steps; ++i) {
        ProductArgs a{};
        a.p = a.q = x;
        a.p_mat = a.q_mat = l.x;
        a.depth = static_cast<int32_t>(l.k);
        a.m = a.n = static_cast<int32_t>(l.n);
        a.to = a.to_turned = gram;
        a.to_mat = l.g;
        a.acc_by = by[i].gram;
        rc = launch_product<kGram>(ctx, a, mats, l.gram_kernel, s);
        if (rc != MQG_OK) return rc;

        a.p = a.q = a.own = gram;
        a.p_mat = a.q_mat = a.own_mat = l.g;
        a.depth = static_cast<int32_t>(l.n);
        a.to = a.to_turned = poly;
        a.acc_by = by[i].poly;
        a.own_by = by[i].poly_own;
        rc = launch_product<kPoly>(ctx, a, mats, l.gram_kernel, s);
        if (rc != MQG_OK) return rc;

        F16 *const now = xt[i & 1], *const then = xt[~i & 1];
        a.acc_by = by[i].x;
        a.own_by = by[i].x_own;
        // B X as it lies, or, for a tall U, its transpose X^T B: rows of the product are rows of U, so that the output is written along its rows
        a.p = tall ? now : poly;
        a.p_mat = tall ? l.x : l.g;
        a.q = tall ? poly : now;
        a.q_mat = tall ? l.g : l.x;
        a.own = tall ? now : x;
        a.own_mat = a.to_mat = l.x;
        a.to = tall ? then : x;
        a.to_turned = tall ? x : then;
        a.m = static_cast<int32_t>(tall ? l.k : l.n);
        a.n = static_cast<int32_t>(tall ? l.n : l.k);
        const bool last = i + 1 == call.steps;
        if (last) {
            a.out = call.out;
            a.out_row = call.out_row;
            a.out_mat = call.out_mat;
            a.out_m = static_cast<int32_t>(rows);
            a.out_n = static_cast<int32_t>(cols);
            a.out_type = call.out_type;
            a.step = call.step;
            a.keep = call.keep;
        }
        rc = last ? launch_product<kOut>(ctx, a, mats, l.x_kernel, s) : launch_product<kIterate>(ctx, a, mats, l.x_kernel, s);
        if (rc != MQG_OK) return rc;
    }
    return MQG_OK;
}

}  // namespace mqg
