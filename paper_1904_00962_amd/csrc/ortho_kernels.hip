// Newton-Schulz orthogonalization of lists of matrices, and the Muon step made of
// it, for gfx950.
//
// With X = G / (||G||_F + eps), an iteration is A = X X^T (or X^T X, on the shorter
// side), P = a I + b A + c A A, X <- P X (or X P): an odd quintic of X's singular
// values. Of A and P, which are symmetric, only tiles on and below the diagonal are
// computed; each is written to its mirror's place too. One launch covers the tiles
// of every matrix of a plan, so an iteration is three launches however many
// matrices there are. Long matrices of lists with much to do iterate on their short side
// in chains (ortho_internal.h).
//
// X, A and P are held in 16-bit floats (11 significant bits; with bfloat16's 8 the result
// for independent entries would be 1e-2 off instead of 1.3e-3), scaled by a power of two;
// sums are fp32. `split`, the default, holds each as the sum of two such numbers and sums
// three products (high high, high low, low high): 22 significant bits, an fp32-grade
// result. The steps multiply small singular values by up to a^steps, and the roundings of
// large ones with them: with one number, up to 0.15 off where one singular value outweighs
// all others, and 6e-5 with two.
#include <hip/hip_runtime.h>
#include <math.h>

#include "lamb_ops.h"
#include "mma_tile.h"
#include "ortho_internal.h"

namespace lamb_mi355x {
namespace {

__device__ inline float widen(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }

__device__ inline uint16_t to_bf16(float v) {
    return __builtin_bit_cast(uint16_t, __bf16(v));
}

__device__ inline uint16_t to_half(float v) {
    return __builtin_bit_cast(uint16_t, _Float16(v));
}

__device__ inline float from_half(uint16_t v) { return float(__builtin_bit_cast(_Float16, v)); }

// Keeps a value as it is in fp32. Without it the compiler takes the high part of a
// product from a fused multiply that rounds once, and subtracts one that rounds
// twice: near a tie the low part then belongs to another high part.
__device__ inline void pin(float &v) { asm volatile("" : "+v"(v)); }

__device__ inline ushort4 high_halves(float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) pin(v[i]);
    return make_ushort4(to_half(v[0]), to_half(v[1]), to_half(v[2]), to_half(v[3]));
}

// What the high parts leave.
__device__ inline ushort4 low_halves(const float (&v)[4], ushort4 hi) {
    return make_ushort4(to_half(v[0] - from_half(hi.x)), to_half(v[1] - from_half(hi.y)),
                        to_half(v[2] - from_half(hi.z)), to_half(v[3] - from_half(hi.w)));
}

// Eight values of a row from column `col`, of which `n` exist; the rest are 0.
template <bool BF16>
__device__ inline void load_row(const void *base, int64_t at, int n, bool vector, float (&v)[8]) {
    if (BF16) {
        const uint16_t *p = (const uint16_t *)base + at;
        if (vector && n == 8) {
            const uint4 w = load_global<uint4>(p);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(u[i] << 16);
                v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? widen(load_global<uint16_t>(p + i)) : 0.0f;
    } else {
        const float *p = (const float *)base + at;
        if (vector && n == 8) {
            const float4 lo = load_global<float4>(p), hi = load_global<float4>(p + 4);
            v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
            v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? load_global<float>(p + i) : 0.0f;
    }
}

__device__ inline void store_row(float *p, int n, bool vector, const float (&v)[8]) {
    if (vector && n == 8) {
        store_global(p, make_float4(v[0], v[1], v[2], v[3]));
        store_global(p + 4, make_float4(v[4], v[5], v[6], v[7]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n)
            store_global(p + i, v[i]);
}

// The workgroup's sum, on every thread of wave 0, in a fixed order.
__device__ inline double block_sum(double v, double *shared) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0)
        shared[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < kNsBlock / 64; ++w) sum += shared[w];
    return sum;
}

// Calls f(row, col, n) for the units of this workgroup: n columns from col of a row.
template <class F>
__device__ inline void for_units(const NsMatrix &mat, F f) {
    const int64_t per_row = mat.ld / 8, units = per_row * mat.rows;
    const int64_t first = int64_t(blockIdx.x - mat.first_block) * kNsBlockUnits;
#pragma unroll
    for (int i = 0; i < kNsUnits; ++i) {
        const int64_t u = first + i * kNsBlock + threadIdx.x;
        if (u < units) {
            int64_t row;
            if (units <= INT32_MAX)
                row = uint32_t(u) / uint32_t(per_row);
            else
                row = u / per_row;
            const int col = int(u - row * per_row) * 8;
            f(row, col, mat.cols - col < 8 ? mat.cols - col : 8);
        }
    }
}

// Raises the flag when a scaled gradient is not finite. Bound by HBM: reads it once.
template <bool BF16>
__global__ __launch_bounds__(kNsBlock) void ns_check_kernel(const NsMatrix *matrices,
                                                            const int32_t *block_matrix,
                                                            float grad_scale, uint32_t *flag) {
    const NsMatrix mat = matrices[block_matrix[blockIdx.x]];
    bool bad = false;
    for_units(mat, [&](int64_t row, int col, int n) {
        float g[8];
        load_row<BF16>(mat.in, row * mat.in_stride + col, n, mat.vector, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) bad |= !isfinite(g[i] * grad_scale);
    });
    if (__any(bad) && (threadIdx.x & 63) == 0)
        atomicOr(flag, 1u);
}

// momentum m + from_grad g, rounded once: in fp64, which costs these passes nothing.
__device__ inline float mix(const NsStep &step, float m, float g) {
    return float(__builtin_fma(step.momentum, double(m), step.from_grad * double(g)));
}

// Each workgroup's sum of squares of the matrix to orthogonalize, in fp64. Muon:
// m <- momentum m + (1 - momentum) g first; the matrix is momentum m + (1 - momentum) g
// (Nesterov) or m. Bound by HBM: 8 B read (6 with bf16 gradients) and 4 written per
// element; BERT-Large's 302M elements with bf16 gradients take 543 us, 5.6 TB/s. Four
// units of 8 columns a thread keep enough loads in flight.
template <bool MUON, bool BF16>
__global__ __launch_bounds__(kNsBlock) void ns_norm_kernel(const NsMatrix *matrices,
                                                           const int32_t *block_matrix,
                                                           NsStep step, double *partials,
                                                           uint32_t *flag,
                                                           int32_t *nonfinite_out) {
    __shared__ double shared[kNsBlock / 64];
    const NsMatrix mat = matrices[block_matrix[blockIdx.x]];
    const bool skip = MUON && flag && flag[0];
    if (MUON && blockIdx.x == 0 && threadIdx.x == 0) {
        if (flag)
            flag[1] = skip;
        if (nonfinite_out)
            *nonfinite_out = skip;
    }
    double sum = 0.0;
    for_units(mat, [&](int64_t row, int col, int n) {
        float g[8];
        load_row<BF16>(mat.in, row * mat.in_stride + col, n, mat.vector, g);
        if (MUON) {
            float m[8];
            float *at = mat.m + row * mat.cols + col;
            load_row<false>(mat.m, row * mat.cols + col, n, mat.vector, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m[i] = mix(step, m[i], g[i]);
                g[i] = step.nesterov ? mix(step, m[i], g[i]) : m[i];
            }
            if (!skip)
                store_row(at, n, mat.vector, m);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += double(g[i]) * double(g[i]);
    });
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0)
        partials[blockIdx.x] = sum;
}

// X = matrix * kNsScale / (norm + eps), columns up to ld set to 0. The norm is summed
// by every workgroup from the matrix's partials, in their order: a launch less. Muon's
// matrix is formed again from m and the gradient, which is cheaper than a copy of it.
// Bound by HBM: 10 B per element of BERT-Large's 302M (split), 579 us, 5.2 TB/s.
template <bool MUON, bool BF16, bool SPLIT>
__global__ __launch_bounds__(kNsBlock) void ns_convert_kernel(const NsMatrix *matrices,
                                                              const int32_t *block_matrix,
                                                              NsStep step,
                                                              const double *partials,
                                                              uint32_t *flag) {
    if (MUON && flag && blockIdx.x == 0 && threadIdx.x == 0)
        flag[0] = 0;
    __shared__ double shared[kNsBlock / 64];
    const NsMatrix mat = matrices[block_matrix[blockIdx.x]];
    double sum = 0.0;
    for (int i = threadIdx.x; i < mat.blocks; i += kNsBlock) sum += partials[mat.first_block + i];
    sum = block_sum(sum, shared);
    // below 2^-100 the quotient may pass fp32's range (eps 0): a power of two goes first
    const double norm = sqrt(sum) + double(step.eps);
    const float first = norm < 0x1p-100 ? 0x1p64f : 1.0f;
    const float to_x = float(double(kNsScale) / (norm * double(first)));
    for_units(mat, [&](int64_t row, int col, int n) {
        float g[8];
        if (!MUON || step.nesterov)
            load_row<BF16>(mat.in, row * mat.in_stride + col, n, mat.vector, g);
        if (MUON) {
            float m[8];
            load_row<false>(mat.m, row * mat.cols + col, n, mat.vector, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = step.nesterov ? mix(step, m[i], g[i]) : m[i];
        }
        uint16_t *x = mat.x[0] + row * mat.ld + col;
        ushort4 hi[2], lo[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = g[4 * h + i] * first * to_x;
            hi[h] = high_halves(v);
            lo[h] = low_halves(v, hi[h]);
        }
        auto pack = [](const ushort4 (&h)[2]) {
            return make_uint4(h[0].x | uint32_t(h[0].y) << 16, h[0].z | uint32_t(h[0].w) << 16,
                              h[1].x | uint32_t(h[1].y) << 16, h[1].z | uint32_t(h[1].w) << 16);
        };
        store_global(x, pack(hi));
        if (SPLIT)
            store_global(x + mat.x_low, pack(lo));
    });
}

__device__ inline Operand rows_of(const uint16_t *p, int64_t ld, int64_t first, int64_t rows) {
    return Operand{(const char *)(p + first * ld), ld * 2, int32_t(rows - first)};
}

__device__ inline Operand columns_of(const uint16_t *p, int64_t ld, int64_t first) {
    return Operand{(const char *)(p + first), ld * 2, int32_t(ld - first)};
}

// A symmetric result's tile, and its mirror image where that is another tile, in
// `parts` 16-bit parts. acc holds the values already; rows and columns from the
// matrix's side on are 0.
template <class Shape>
__device__ inline void store_symmetric(const NsMatrix &mat, uint16_t *to, const NsTile &tile,
                                       float4v (&acc)[Shape::MI][Shape::NI], short *lds) {
    static_assert(Shape::BM == Shape::BN, "square tiles");
    const Place<Shape> at;
    const TileStore<Shape::BM, Shape::BN, Shape::kThreads> store(lds);
    const int64_t ld = mat.side_ld;
    const int m0 = tile.row * Shape::BM, n0 = tile.col * Shape::BN;
#pragma unroll
    for (int part = 0; part < Shape::PARTS; ++part) {
        uint16_t *plane = to + part * mat.gram_low;
        auto each = [&](auto put) {
#pragma unroll
            for (int i = 0; i < Shape::MI; ++i)
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j) {
                    float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    ushort4 h = high_halves(v);
                    if (part)
                        h = low_halves(v, h);
                    put(at.row + 16 * i, at.col + 16 * j, h);
                }
        };
        each([&](int m, int n, ushort4 h) { store.put(m, n, h); });
        store.template flush<false>(plane + m0 * ld + n0, ld, mat.side - m0, mat.side_ld - n0);
        if (tile.row != tile.col) {
            each([&](int m, int n, ushort4 h) { store.put_mirror(m, n, h); });
            store.template flush<true>(plane + n0 * ld + m0, ld, mat.side - n0, mat.side_ld - m0);
        }
    }
}

// A = X X^T or X^T X, tiles on and below the diagonal, the sum over the long side. Bound
// by the matrix cores. BERT-Large's 144 matrices, split: 1.11 ms for 0.93e12 16-bit
// operations, symmetric halves counted once (0.83 PFLOP/s; 1.04 counting whole tiles on
// the diagonal); six layers of width 1600, 16-bit, 0.39 ms, 0.75 (1.07 with partial tiles).
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void ns_gram_kernel(
    const NsMatrix *matrices, const NsTile *tiles, NsTurn turn) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const NsTile tile = tiles[blockIdx.x];
    const NsMatrix mat = matrices[tile.matrix];
    const uint16_t *x = (mat.chain ? turn.parity[1] : turn.parity[0]) ? mat.x[1] : mat.x[0];
    float4v acc[Shape::MI][Shape::NI] = {};
    const int64_t m = int64_t(tile.row) * Shape::BM, n = int64_t(tile.col) * Shape::BN;
    if (mat.tall) {
        const Operand a = columns_of(x, mat.ld, m);
        const Operand b = columns_of(x, mat.ld, n);
        tile_product<HalfMath, Shape, true, true>(acc, lds, a, b, mat.rows, 2 * mat.x_low,
                                                   2 * mat.x_low);
    } else {
        const Operand a = rows_of(x, mat.ld, m, mat.rows);
        const Operand b = rows_of(x, mat.ld, n, mat.rows);
        tile_product<HalfMath, Shape, false, false>(acc, lds, a, b, mat.cols, 2 * mat.x_low,
                                                   2 * mat.x_low);
    }
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i)
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) acc[i][j] *= 1.0f / kNsScale;
    store_symmetric<Shape>(mat, mat.gram[0], tile, acc, lds);
}

// P = a I + b A + c A A, likewise; A's own tile is added from memory at the end. BERT-Large,
// split: 0.69 ms, 0.67 PFLOP/s (0.84): sums over 1024 only, so a tile's fixed part and the
// last round weigh more.
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void ns_poly_kernel(
    const NsMatrix *matrices, const NsTile *tiles, NsTurn turn, NsStep step) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const NsTile tile = tiles[blockIdx.x];
    const NsMatrix mat = matrices[tile.matrix];
    const bool odd = mat.chain && (turn.turn & 1);
    const uint16_t *gram = odd ? mat.gram[1] : mat.gram[0];
    float4v acc[Shape::MI][Shape::NI] = {};
    const Operand a = rows_of(gram, mat.side_ld, int64_t(tile.row) * Shape::BM, mat.side);
    const Operand b = rows_of(gram, mat.side_ld, int64_t(tile.col) * Shape::BN, mat.side);
    tile_product<HalfMath, Shape, false, false>(acc, lds, a, b, mat.side, 2 * mat.gram_low,
                                                   2 * mat.gram_low);
    const Place<Shape> at;
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i) {
        const int m = tile.row * Shape::BM + at.row + 16 * i;
        // a row's loads go out together: from inside the matrix, wherever they are used
        ushort4 part[Shape::PARTS][Shape::NI];
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) {
            const int n = tile.col * Shape::BN + at.col + 16 * j;
            const uint16_t *from = gram + int64_t(m < mat.side ? m : mat.side - 1) * mat.side_ld +
                                   (n < mat.side_ld ? n : mat.side_ld - 4);
#pragma unroll
            for (int p = 0; p < Shape::PARTS; ++p)
                part[p][j] = load_global<ushort4>(from + p * mat.gram_low);
        }
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) {
            const int n = tile.col * Shape::BN + at.col + 16 * j;
            float g[4] = {from_half(part[0][j].x), from_half(part[0][j].y),
                          from_half(part[0][j].z), from_half(part[0][j].w)};
            if (Shape::PARTS == 2) {
                const ushort4 lo = part[Shape::PARTS - 1][j];
                g[0] += from_half(lo.x), g[1] += from_half(lo.y);
                g[2] += from_half(lo.z), g[3] += from_half(lo.w);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = __builtin_fmaf(step.b, g[r], step.c * (acc[i][j][r] * (1.0f / kNsScale)));
                if (m == n + r)
                    v = __builtin_fmaf(step.a, kNsScale, v);
                // rows and columns from `side` on are 0
                acc[i][j][r] = m < mat.side && n + r < mat.side ? v : 0.0f;
            }
        }
    }
    store_symmetric<Shape>(mat, odd ? mat.poly[1] : mat.poly[0], tile, acc, lds);
}

// Q, T and the next A of a chain, like ns_poly_kernel. Q and T of an iteration are one
// launch: neither alone fills the card (BERT-Large's 48 chained matrices have 480 tiles
// in a product).
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void ns_product_kernel(
    const NsMatrix *matrices, const NsTile *tiles, NsTurn turn) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const NsTile tile = tiles[blockIdx.x];
    const NsMatrix mat = matrices[tile.matrix];
    const bool odd = turn.turn & 1;
    uint16_t *const p = odd ? mat.poly[1] : mat.poly[0];
    uint16_t *const p_before = odd ? mat.poly[0] : mat.poly[1];
    const uint16_t *left = p, *right;
    uint16_t *out;
    float back = 1.0f / kNsScale;
    if (tile.product == kNsQ) {
        // turn 1: q = P_1 P_0; turn 2: P_2 q, where P_1 was
        right = turn.turn == 1 ? p_before : mat.q;
        out = turn.turn == 1 ? mat.q : p_before;
        back = turn.turn == 1 ? kNsQScale / (kNsScale * kNsScale) : 1.0f / kNsScale;
    } else if (tile.product == kNsT) {
        right = odd ? mat.gram[1] : mat.gram[0];
        out = mat.t;
    } else {
        left = mat.t;
        right = p;
        out = odd ? mat.gram[0] : mat.gram[1];
    }
    float4v acc[Shape::MI][Shape::NI] = {};
    tile_product<HalfMath, Shape, false, false>(
        acc, lds, rows_of(left, mat.side_ld, int64_t(tile.row) * Shape::BM, mat.side),
        rows_of(right, mat.side_ld, int64_t(tile.col) * Shape::BN, mat.side), mat.side,
        2 * mat.gram_low, 2 * mat.gram_low);
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i)
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) acc[i][j] *= back;
    store_symmetric<Shape>(mat, out, tile, acc, lds);
}

__device__ inline float update_scale(const NsMatrix &mat, int32_t kind) {
    if (kind == LAMB_MUON_RMS)
        return 0.2f * sqrtf(float(mat.rows > mat.cols ? mat.rows : mat.cols));
    if (kind == LAMB_MUON_SPECTRAL)
        return mat.tall ? sqrtf(float(mat.rows) / float(mat.cols)) : 1.0f;
    return 1.0f;
}

// X <- P X (Q X, X P): the largest product, bound by the matrix cores. BERT-Large, split,
// all matrices: 1.77 ms for 1.86e12 16-bit operations, 1.05 PFLOP/s; the last one, which
// moves the parameters (8 B per element) in its epilogue, 1.93 ms. Six layers of width
// 1600, 16-bit: 0.63 ms, 0.94 (1.18 with partial tiles).
template <class Shape, int KIND>  // KIND: an NsKind, or -1 for the other X
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void ns_update_kernel(
    const NsMatrix *matrices, const NsTile *tiles, NsTurn turn, NsStep step,
    const uint32_t *flag) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const NsTile tile = tiles[blockIdx.x];
    const NsMatrix mat = matrices[tile.matrix];
    if (KIND == kNsMuon && flag && flag[1])
        return;
    const int parity = mat.chain ? turn.parity[1] : turn.parity[0];
    const uint16_t *x = parity ? mat.x[1] : mat.x[0];
    const bool chained = mat.chain && turn.turn > 0;
    const uint16_t *q = !chained ? mat.poly[0] : turn.turn == 1 ? mat.q : mat.poly[1];
    float4v acc[Shape::MI][Shape::NI] = {};
    const int64_t m0 = int64_t(tile.row) * Shape::BM, n0 = int64_t(tile.col) * Shape::BN;
    if (mat.tall) {
        const Operand a = rows_of(x, mat.ld, m0, mat.rows);
        const Operand b = rows_of(q, mat.side_ld, n0, mat.side);
        tile_product<HalfMath, Shape, false, false>(acc, lds, a, b, mat.side, 2 * mat.x_low,
                                                   2 * mat.gram_low);
    } else {
        const Operand a = rows_of(q, mat.side_ld, m0, mat.side);
        const Operand b = columns_of(x, mat.ld, n0);
        tile_product<HalfMath, Shape, false, true>(acc, lds, a, b, mat.side, 2 * mat.gram_low,
                                                   2 * mat.x_low);
    }
    const Place<Shape> at;
    const float back = (KIND < 0 ? 1.0f : 1.0f / kNsScale) / (chained ? kNsQScale : kNsScale);
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i)
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) acc[i][j] *= back;
    if (KIND < 0 || (KIND == kNsBf16Out && mat.vector && mat.cols % 8 == 0)) {
        const TileStore<Shape::BM, Shape::BN, Shape::kThreads> store(lds);
        uint16_t *to = KIND < 0 ? (parity ? mat.x[0] : mat.x[1]) : (uint16_t *)mat.out;
        const int64_t ld = KIND < 0 ? int64_t(mat.ld) : mat.out_stride;
        uint16_t *out = to + m0 * ld + n0;
#pragma unroll
        for (int part = 0; part < (KIND < 0 ? Shape::PARTS : 1); ++part) {
#pragma unroll
            for (int i = 0; i < Shape::MI; ++i)
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j) {
                    float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    ushort4 h;
                    if (KIND < 0) {
                        h = high_halves(v);
                        if (part)
                            h = low_halves(v, h);
                    } else {
                        h = make_ushort4(to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]),
                                         to_bf16(v[3]));
                    }
                    store.put(at.row + 16 * i, at.col + 16 * j, h);
                }
            store.template flush<false>(out + part * mat.x_low, ld, int(mat.rows - m0),
                                        int((KIND < 0 ? mat.ld : mat.cols) - n0));
        }
        return;
    }
    const float move = KIND == kNsMuon ? -step.lr * update_scale(mat, step.scale) : 0.0f;
    const float keep = KIND == kNsMuon && mat.wd ? step.decay : 1.0f;
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i) {
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) {
            const int64_t m = m0 + at.row + 16 * i;
            const int n = int(n0) + at.col + 16 * j;
            if (m >= mat.rows || n >= mat.cols)
                continue;
            float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            const bool whole = mat.vector && n + 4 <= mat.cols;
            if (KIND == kNsBf16Out) {
                uint16_t *out = (uint16_t *)mat.out + m * mat.out_stride + n;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n + r < mat.cols)
                        store_global(out + r, to_bf16(v[r]));
                continue;
            }
            float *out = (float *)mat.out + m * mat.out_stride + n;
            if (KIND == kNsMuon) {
                float xs[4] = {};
                if (whole) {
                    const float4 t = load_global<float4>(out);
                    xs[0] = t.x, xs[1] = t.y, xs[2] = t.z, xs[3] = t.w;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        xs[r] = n + r < mat.cols ? load_global<float>(out + r) : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = __builtin_fmaf(move, v[r], keep * xs[r]);
            }
            if (whole) {
                store_global(out, make_float4(v[0], v[1], v[2], v[3]));
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n + r < mat.cols)
                        store_global(out + r, v[r]);
            }
        }
    }
}

// The shapes of launch_ns_*: see the table in ortho_internal.h.
using Tiny = TileShape<64, 64, 2, 2, 64, 4, 1>;
using Small = TileShape<128, 128, 2, 2, 32, 4, 1>;
using Large = TileShape<256, 256, 2, 4, 32, 4, 1>;
using TinySplit = TileShape<64, 64, 2, 2, 32, 4, 2>;
using SmallSplit = TileShape<128, 128, 2, 2, 32, 2, 2>;
using LargeSplit = TileShape<256, 256, 2, 4, 32, 2, 2>;

}  // namespace

hipError_t launch_ns_check(const NsMatrix *matrices, const int32_t *block_matrix, int32_t blocks,
                           bool bf16_in, float grad_scale, uint32_t *flag, hipStream_t stream) {
    auto kernel = bf16_in ? ns_check_kernel<true> : ns_check_kernel<false>;
    kernel<<<blocks, kNsBlock, 0, stream>>>(matrices, block_matrix, grad_scale, flag);
    return hipGetLastError();
}

hipError_t launch_ns_norms(const NsMatrix *matrices, const int32_t *block_matrix, int32_t blocks,
                           bool muon, bool bf16_in, const NsStep &step, double *partials,
                           uint32_t *flag, int32_t *nonfinite_out, hipStream_t stream) {
    auto kernel = muon ? (bf16_in ? ns_norm_kernel<true, true> : ns_norm_kernel<true, false>)
                       : (bf16_in ? ns_norm_kernel<false, true> : ns_norm_kernel<false, false>);
    kernel<<<blocks, kNsBlock, 0, stream>>>(matrices, block_matrix, step, partials, flag,
                                            nonfinite_out);
    return hipGetLastError();
}

hipError_t launch_ns_convert(const NsMatrix *matrices, const int32_t *block_matrix,
                             int32_t blocks, bool muon, bool bf16_in, bool split,
                             const NsStep &step, const double *partials, uint32_t *flag,
                             hipStream_t stream) {
    auto pick = [&](auto split_c) {
        constexpr bool S = decltype(split_c)::value;
        return muon ? (bf16_in ? ns_convert_kernel<true, true, S>
                               : ns_convert_kernel<true, false, S>)
                    : (bf16_in ? ns_convert_kernel<false, true, S>
                               : ns_convert_kernel<false, false, S>);
    };
    auto kernel = split ? pick(std::true_type{}) : pick(std::false_type{});
    kernel<<<blocks, kNsBlock, 0, stream>>>(matrices, block_matrix, step, partials, flag);
    return hipGetLastError();
}

namespace {

template <class F>
hipError_t with_shape(int shape, bool split, F f) {
    switch (split ? 8 + shape : shape) {
    case kNsTiny: f(Tiny{}); break;
    case kNsSmall: f(Small{}); break;
    case kNsLarge: f(Large{}); break;
    case 8 + kNsTiny: f(TinySplit{}); break;
    case 8 + kNsSmall: f(SmallSplit{}); break;
    case 8 + kNsLarge: f(LargeSplit{}); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ns_gram(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                          bool split, const NsTurn &turn, hipStream_t stream) {
    return with_shape(shape, split, [&](auto s) {
        using Shape = decltype(s);
        ns_gram_kernel<Shape><<<n, Shape::kThreads, 0, stream>>>(matrices, tiles, turn);
    });
}

hipError_t launch_ns_product(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                             bool split, const NsTurn &turn, hipStream_t stream) {
    return with_shape(shape, split, [&](auto s) {
        using Shape = decltype(s);
        ns_product_kernel<Shape><<<n, Shape::kThreads, 0, stream>>>(matrices, tiles, turn);
    });
}

hipError_t launch_ns_poly(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                          bool split, const NsTurn &turn, const NsStep &step,
                          hipStream_t stream) {
    return with_shape(shape, split, [&](auto s) {
        using Shape = decltype(s);
        ns_poly_kernel<Shape><<<n, Shape::kThreads, 0, stream>>>(matrices, tiles, turn, step);
    });
}

hipError_t launch_ns_update(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                            bool split, const NsTurn &turn, bool last, NsKind kind,
                            const NsStep &step, const uint32_t *flag, hipStream_t stream) {
    return with_shape(shape, split, [&](auto s) {
        using Shape = decltype(s);
        auto kernel = !last ? ns_update_kernel<Shape, -1>
                      : kind == kNsBf16Out ? ns_update_kernel<Shape, kNsBf16Out>
                      : kind == kNsF32Out  ? ns_update_kernel<Shape, kNsF32Out>
                                           : ns_update_kernel<Shape, kNsMuon>;
        kernel<<<n, Shape::kThreads, 0, stream>>>(matrices, tiles, turn, step, flag);
    });
}

}  // namespace lamb_mi355x
