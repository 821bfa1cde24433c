// Softmax cross entropy of hidden states H (tokens x dim, bf16) against a vocabulary
// table W (vocab x dim, bf16), and its gradients, for gfx950, without keeping the
// logits L = H W^T.
//
// Forward: tiles of L stay in registers; of each only its rows' maximum and sum of
// exponentials (and the target's logit) leave, and a second pass joins them into
// lse_i = log sum_v exp L_iv. Backward, per piece of the vocabulary: L's tiles again,
// now as Q = exp(L - lse) - [v = target] in bf16, then dH += Q W and dW = Q^T H, each
// scaled once in fp32 at its end. So 8 tokens dim vocab operations are done where
// keeping L would need 6, for a workspace of one piece of Q.
//
// Tokens that do not count (ignore_index) are left out before anything is computed:
// the rows that do are packed together, and how many there are stays on the device,
// where a tile past them ends at once. What such a token's row holds, NaN included,
// reaches no result.
//
// Q's rounding to bf16 (2^-8 at most, relative, each entry by itself) is the one to
// fewer bits; sums are fp32. It is as large as the rounding of a bf16 gradient: 8192 tokens
// of 64 columns against 500 words end 2.4e-3 off, 1.7e-3 by the result's rounding alone;
// 1229 against 30522 words, where few words carry the sums, 1.66e-3 and 1.66e-3. An fp32
// gradient of the table is promised more, and gets Q in two parts (2^-16) for a product more.
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "mma_tile.h"
#include "ops_host.h"
#include "xent_internal.h"

namespace lamb_mi355x {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kXcdCount = 8;
constexpr int kGroupRows = 8;  // tile rows that are worked on together

using Tiny = TileShape<64, 64, 2, 2, 64, 4, 1>;
using Small = TileShape<128, 128, 2, 2, 32, 4, 1>;
using Large = TileShape<256, 256, 2, 4, 32, 4, 1>;

__device__ inline uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, __bf16(v)); }
__device__ inline float widen(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }

// The workgroup's tile of rows x cols tiles. Workgroups go to the dies in turn; each
// die gets a run of tiles, kGroupRows rows tall, that share operand rows in its L2.
struct TileAt {
    int row, col;  // row >= rows: none
    __device__ TileAt(int rows, int cols) {
        const uint32_t n = uint32_t(rows) * uint32_t(cols);
        const uint32_t b = blockIdx.y * gridDim.x + blockIdx.x;
        if (b >= n) {
            row = rows, col = 0;
            return;
        }
        const uint32_t die = b % kXcdCount, each = n / kXcdCount, more = n % kXcdCount;
        const uint32_t item = die * each + (die < more ? die : more) + b / kXcdCount;
        const uint32_t band = item / (kGroupRows * cols), in = item % (kGroupRows * cols);
        const int first = int(band) * kGroupRows;
        const int tall = rows - first < kGroupRows ? rows - first : kGroupRows;
        row = first + int(in) % tall;
        col = int(in) / tall;
    }
};

__host__ __device__ inline int tiles_of(int n, int tile) { return (n + tile - 1) / tile; }

__device__ inline Operand rows_at(const uint16_t *p, int64_t ld, int64_t first, int32_t rows) {
    return Operand{(const char *)(p + first * ld), ld * 2, int32_t(rows - first)};
}

__device__ inline Operand columns_at(const uint16_t *p, int64_t ld, int32_t first, int32_t extent) {
    return Operand{(const char *)(p + first), ld * 2, extent - first};
}

__device__ inline int64_t target_of(const XentPack &a, int64_t i) {
    return a.wide ? ((const int64_t *)a.targets)[i] : int64_t(((const int32_t *)a.targets)[i]);
}

__device__ inline void copy_row(const uint16_t *src, uint16_t *dst, int dim, int ld, bool vector,
                                int lane) {
    for (int c = lane * 8; c < ld; c += 64 * 8) {
        if (vector && c + 8 <= dim) {
            *(uint4 *)(dst + c) = *(const uint4 *)(src + c);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[c + i] = c + i < dim ? src[c + i] : uint16_t(0);
        }
    }
}

// Each workgroup counts the tokens before its own that count (from L2: 8 bytes each),
// so that one launch packs in order. Bound by latency for few tokens (2.8 us for 7) and
// by memory: 8192 tokens of 1600 take 20 us, of which the copy needs 10.
__global__ __launch_bounds__(256) void xent_pack_kernel(XentPack a) {
    __shared__ int32_t before[4];
    __shared__ int32_t row_of[kPackTokens];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t begin = int64_t(blockIdx.x) * kPackTokens * a.rounds;
    int32_t count = 0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < begin; i += 256) count += target_of(a, i) != a.ignore;
#pragma unroll
    for (int d = 32; d; d >>= 1) count += __shfl_xor(count, d);
    if (lane == 0)
        before[wave] = count;
    __syncthreads();
    int32_t base = before[0] + before[1] + before[2] + before[3];
    for (int32_t round = 0; round < a.rounds; ++round) {
        const int64_t first = begin + int64_t(round) * kPackTokens;
        if (first >= a.tokens && first > 0)
            return;
        if (wave == 0) {
            const int64_t i = first + lane;
            const int64_t t = i < a.tokens ? target_of(a, i) : a.ignore;
            const bool counts = lane < kPackTokens && t != a.ignore;
            const uint64_t mask = __ballot(counts);
            const int32_t row = base + __popcll(mask & ((uint64_t(1) << lane) - 1));
            if (lane < kPackTokens)
                row_of[lane] = counts ? row : -1;
            if (counts) {
                a.source[row] = int32_t(i);
                a.target[row] = t >= 0 && t < a.vocab ? int32_t(t) : -1;
            } else if (lane < kPackTokens && i < a.tokens && a.loss) {
                a.loss[i] = 0.0f;
                a.lse[i] = 0.0f;
            }
            base += __popcll(mask);
            if (first + kPackTokens >= a.tokens && lane == 0)
                *a.kept = base;
        }
        __syncthreads();
        for (int t = wave; t < kPackTokens && first + t < a.tokens; t += 4) {
            if (row_of[t] >= 0) {
                copy_row(a.hidden + (first + t) * a.stride, a.packed + int64_t(row_of[t]) * a.ld,
                         a.dim, a.ld, a.vector, lane);
            } else if (a.grad_hidden) {
                uint16_t *out = a.grad_hidden + (first + t) * a.grad_stride;
                for (int c = lane; c < a.dim; c += 64) out[c] = 0;
            }
        }
        __syncthreads();
    }
}

// For tables whose rows the product cannot read in place: unaligned, or dim not a multiple
// of 8. Bound by HBM.
__global__ __launch_bounds__(256) void xent_copy_kernel(const uint16_t *src, int64_t stride,
                                                        uint16_t *dst, int32_t dim, int32_t ld,
                                                        int64_t rows) {
    const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row < rows)
        copy_row(src + row * stride, dst + row * ld, dim, ld, false, threadIdx.x & 63);
}

template <class Shape>
__device__ inline void logits_tile(float4v (&acc)[Shape::MI][Shape::NI], const short *lds,
                                   const XentArgs &a, int64_t m0, int64_t n0, int32_t kept) {
    tile_product<Bf16Math, Shape, false, false>(acc, lds, rows_at(a.hidden, a.ld, m0, kept),
                                                rows_at(a.table, a.table_ld, n0, a.vocab), a.dim);
}

// Joins two (maximum, sum of exponentials from it).
__device__ inline float2 join(float2 p, float2 q) {
    const float top = fmaxf(p.x, q.x);
    const float from = top == -INFINITY ? 0.0f : top;
    return make_float2(top, p.y * __builtin_amdgcn_exp2f((p.x - from) * kLog2e) +
                                q.y * __builtin_amdgcn_exp2f((q.x - from) * kLog2e));
}

// A tile of logits, its rows' maxima and sums of exponentials: in registers, then over the
// 4 lanes of a row, then over the WN waves through LDS. Bound by the matrix cores: 8192
// tokens of 1600 against 50257 words take 1.15 ms, 1.15 PFLOP/s; 1190 of 1024 against 30522
// (9.3 rows of 128 x 128 tiles) 0.12, 0.62.
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void xent_logits_kernel(
    XentArgs a, float2 *parts, float *at_target) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const int32_t kept = *a.kept;
    const TileAt tile(tiles_of(a.tokens, Shape::BM), tiles_of(a.vocab, Shape::BN));
    const int m0 = tile.row * Shape::BM, n0 = tile.col * Shape::BN;
    if (m0 >= kept)
        return;
    float4v acc[Shape::MI][Shape::NI] = {};
    logits_tile<Shape>(acc, lds, a, m0, n0, kept);
    const Place<Shape> at;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float2 *row_parts = (float2 *)lds;  // [BM][WN]
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i) {
        const int m = m0 + at.row + 16 * i;
        const int target = m < kept ? a.target[m] : -1;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = n0 + at.col + 16 * j + r;
                const float v = acc[i][j][r];
                if (n < a.vocab)
                    top = fmaxf(top, v);
                if (n == target)
                    at_target[m] = v;
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // no column of this wave exists, or all are -inf: any finite offset will do
        const float from = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = n0 + at.col + 16 * j + r;
                const float e = __builtin_amdgcn_exp2f((acc[i][j][r] - from) * kLog2e);
                sum += n < a.vocab ? e : 0.0f;
            }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16)
            row_parts[(at.row + 16 * i) * Shape::WN + wave % Shape::WN] = make_float2(top, sum);
    }
    __syncthreads();
    for (int t = threadIdx.x; t < Shape::BM && m0 + t < kept; t += Shape::kThreads) {
        float2 sum = row_parts[t * Shape::WN];
        for (int w = 1; w < Shape::WN; ++w) sum = join(sum, row_parts[t * Shape::WN + w]);
        parts[int64_t(tile.col) * a.tokens + m0 + t] = sum;
    }
}

// kReduceTokens tokens by 16 threads each, joined in a fixed order. `mean` non-null: of
// all tokens, which are one workgroup's. Bound by latency: 8 us for 8192 tokens of 197
// parts each (13 MB).
__global__ __launch_bounds__(256) void xent_reduce_kernel(XentArgs a, int32_t n_parts,
                                                          const float2 *parts,
                                                          const float *at_target, float *loss,
                                                          float *lse, float *mean) {
    __shared__ float2 shared[16][kReduceTokens];
    const int32_t kept = *a.kept;
    const int t = threadIdx.x % kReduceTokens, group = threadIdx.x / kReduceTokens;
    const int m = blockIdx.x * kReduceTokens + t;
    if (int(blockIdx.x) * kReduceTokens >= kept) {
        if (mean && threadIdx.x == 0)
            *mean = 0.0f;
        return;
    }
    float2 sum = make_float2(-INFINITY, 0.0f);
    if (m < kept)
        for (int p = group; p < n_parts; p += 16) sum = join(sum, parts[int64_t(p) * a.tokens + m]);
    shared[group][t] = sum;
    __syncthreads();
    double value = 0.0;
    if (group == 0 && m < kept) {
        for (int g = 1; g < 16; ++g) sum = join(sum, shared[g][t]);
        const int token = a.source[m];
        const bool inside = a.target[m] >= 0;
        // the loss not from lse, whose last place is that of the largest logit: a token whose
        // target is far ahead has a loss much smaller than that
        const float rest = logf(sum.y);
        const float mine = inside ? (sum.x - at_target[m]) + rest : NAN;
        lse[token] = inside ? sum.x + rest : NAN;
        loss[token] = mine;
        value = mine;
    }
    if (mean && group < 4) {  // wave 0, whose other groups hold zeros
#pragma unroll
        for (int d = 8; d; d >>= 1) value += __shfl_xor(value, d);
        if (threadIdx.x == 0)
            *mean = float(value / double(kept));
    }
}

// One workgroup, so that the sum has one order: 4.6 us for 8192 losses.
__global__ __launch_bounds__(1024) void xent_mean_kernel(const float *loss, int32_t tokens,
                                                         const int32_t *kept, float *mean) {
    __shared__ double shared[16];
    double sum = 0.0;
    for (int i = threadIdx.x; i < tokens; i += 1024) sum += double(loss[i]);
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0)
        shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) sum += shared[w];
        const int32_t n = *kept;
        *mean = float(sum / double(n > 1 ? n : 1));
    }
}

// Q of a piece: the logits again, so the same product, and 2 B written per entry, through
// LDS in whole lines (128 x 128 tiles, 1190 tokens of 1024 against 30522 words: 128 us,
// 132 from registers; 256 x 256, 8192 of 1600 against a sixth of 50257: 245 and 240).
// Bound by the matrix cores: 0.58 and 0.90 PFLOP/s.
// LOW: the rest of each entry too, a plane of its own.
template <class Shape, bool LOW>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void xent_probs_kernel(
    XentArgs a, XentPiece piece, const float *lse) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const int32_t kept = *a.kept;
    const TileAt tile(tiles_of(a.tokens, Shape::BM), tiles_of(piece.ld, Shape::BN));
    const int m0 = tile.row * Shape::BM, n0 = tile.col * Shape::BN;
    if (m0 >= kept)
        return;
    float4v acc[Shape::MI][Shape::NI] = {};
    logits_tile<Shape>(acc, lds, a, m0, int64_t(piece.first) + n0, kept);
    const Place<Shape> at;
    const TileStore<Shape::BM, Shape::BN, Shape::kThreads> store(lds);
#pragma unroll 1
    for (int part = 0; part <= int(LOW); ++part) {
#pragma unroll
        for (int i = 0; i < Shape::MI; ++i) {
            const int m = m0 + at.row + 16 * i;
            const int target = m < kept ? a.target[m] - piece.first : -1;
            const float from = m < kept ? lse[a.source[m]] : 0.0f;
#pragma unroll
            for (int j = 0; j < Shape::NI; ++j) {
                const int n = n0 + at.col + 16 * j;
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    v[r] = __builtin_amdgcn_exp2f((acc[i][j][r] - from) * kLog2e);
                    v[r] = n + r == target ? v[r] - 1.0f : v[r];
                    v[r] = n + r < piece.count ? v[r] : 0.0f;
                    if (LOW && part)
                        v[r] -= widen(to_bf16(v[r]));
                }
                store.put(at.row + 16 * i, at.col + 16 * j,
                          make_ushort4(to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]),
                                       to_bf16(v[3])));
            }
        }
        uint16_t *plane = LOW && part ? piece.low : piece.probs;
        store.template flush<false>(plane + int64_t(m0) * piece.ld + n0, piece.ld, kept - m0,
                                    piece.ld - n0);
    }
}

// dH += Q W over a piece, in fp32; few rows split the piece's columns over workgroups, each
// with a partial sum of its own. Bound by the matrix cores: 8192 tokens of 1600 against a
// sixth of 50257 words take 199 us, 1.10 PFLOP/s; 7 tokens of 256 against 2003 words 4.4.
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void xent_hidden_kernel(
    XentArgs a, XentPiece piece, int32_t splits, bool add, float *partial) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const int32_t kept = *a.kept;
    const int rows = tiles_of(a.tokens, Shape::BM);
    const TileAt tile(rows * splits, tiles_of(a.dim, Shape::BN));
    const int split = tile.row / rows;
    const int m0 = tile.row % rows * Shape::BM, n0 = tile.col * Shape::BN;
    if (m0 >= kept)
        return;
    // the split's share of the piece, in multiples of 64
    const int share = (tiles_of(piece.count, 64) + splits - 1) / splits * 64;
    const int k0 = split * share;
    const int depth = piece.count - k0 < share ? piece.count - k0 : share;
    float4v acc[Shape::MI][Shape::NI] = {};
    if (depth > 0) {
        Operand q = rows_at(piece.probs, piece.ld, m0, kept);
        q.base += int64_t(k0) * 2;
        const Operand w = columns_at(a.table + (int64_t(piece.first) + k0) * a.table_ld, a.table_ld,
                                     n0, int32_t(a.ld));
        tile_product<Bf16Math, Shape, false, true>(acc, lds, q, w, depth);
    }
    const Place<Shape> at;
    float *out = partial + int64_t(split) * a.tokens * a.ld;
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i) {
        const int m = m0 + at.row + 16 * i;
        if (m >= kept)
            continue;
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) {
            const int n = n0 + at.col + 16 * j;
            if (n >= a.ld)
                continue;
            float4 *to = (float4 *)(out + int64_t(m) * a.ld + n);
            float4 v = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
            if (add) {
                const float4 old = *to;
                v.x += old.x, v.y += old.y, v.z += old.z, v.w += old.w;
            }
            *to = v;
        }
    }
}

__device__ inline float final_scale(const float *grad_loss, float grad_scale, bool mean,
                                    int32_t kept) {
    float s = grad_loss ? *grad_loss * grad_scale : grad_scale;
    return mean ? s / float(kept > 1 ? kept : 1) : s;
}

// The partial sums of dH, in their order, scaled, to the tokens' rows. Bound by HBM: 16 us
// for 8192 x 1600 (79 MB).
__global__ __launch_bounds__(256) void xent_hidden_out_kernel(XentArgs a, int32_t splits,
                                                              const float *partial,
                                                              const float *grad_loss,
                                                              float grad_scale, bool mean,
                                                              uint16_t *grad_hidden,
                                                              int64_t stride) {
    const int32_t kept = *a.kept;
    const int across = tiles_of(a.dim, 1024);
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x;
    const int m = int(block / across);
    const int n = (int(block % across) * 256 + threadIdx.x) * 4;
    if (m >= kept || n >= a.dim)
        return;
    const float scale = final_scale(grad_loss, grad_scale, mean, kept);
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < splits; ++s) {
        const float4 v = *(const float4 *)(partial + (int64_t(s) * a.tokens + m) * a.ld + n);
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
    uint16_t *out = grad_hidden + int64_t(a.source[m]) * stride + n;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (n + r < a.dim)
            out[r] = to_bf16(v[r] * scale);
}

// dW's rows of a piece = Q^T H, the sum over the tokens that count, in chains of
// kChainTokens. Both operands are read transposed from LDS. Bound by the matrix cores: 208 us
// for a sixth of 50257 words, 8192 tokens of 1600, 1.06 PFLOP/s. An fp32 result takes the
// products with both parts of Q.
template <class Shape, bool BF16, bool ADD>
__global__ __launch_bounds__(Shape::kThreads, Shape::kPerCu) void xent_table_kernel(
    XentArgs a, XentPiece piece, const float *grad_loss, float grad_scale, bool mean,
    void *grad_table, int64_t stride, bool vector, float *partial) {
    __shared__ __align__(1024) short lds[Shape::kLds];
    const int32_t kept = *a.kept;
    const TileAt tile(tiles_of(piece.count, Shape::BM), tiles_of(a.dim, Shape::BN));
    const int m0 = tile.row * Shape::BM, n0 = tile.col * Shape::BN;
    const Place<Shape> at;
    float4v acc[Shape::MI][Shape::NI] = {};
#pragma unroll 1
    for (int32_t k0 = 0; k0 < kept; k0 += kChainTokens) {
        const int32_t depth = kept - k0 < kChainTokens ? kept - k0 : kChainTokens;
#pragma unroll 1
        for (int part = BF16 ? 1 : 0; part < 2; ++part) {  // small products first
            const uint16_t *q = (part ? piece.probs : piece.low) + int64_t(k0) * piece.ld;
            tile_product<Bf16Math, Shape, true, true>(
                acc, lds, columns_at(q, piece.ld, m0, piece.ld),
                columns_at(a.hidden + int64_t(k0) * a.ld, a.ld, n0, int32_t(a.ld)), depth);
        }
        if (kept <= kChainTokens)
            break;
        // the chains before are in memory; the last one's sum stays in registers
        const bool last = k0 + depth == kept;
#pragma unroll
        for (int i = 0; i < Shape::MI; ++i) {
            const int m = m0 + at.row + 16 * i;
#pragma unroll
            for (int j = 0; j < Shape::NI; ++j) {
                const int n = n0 + at.col + 16 * j;
                if (m >= piece.count || n >= a.ld)
                    continue;
                float4v *sum = (float4v *)(partial + int64_t(m) * a.ld + n);
                if (k0 > 0)
                    acc[i][j] += *sum;
                if (!last) {
                    *sum = acc[i][j];
                    acc[i][j] = float4v{};
                }
            }
        }
    }
    const float scale = final_scale(grad_loss, grad_scale, mean, kept);
#pragma unroll
    for (int i = 0; i < Shape::MI; ++i) {
        const int m = m0 + at.row + 16 * i;
        if (m >= piece.count)
            continue;
#pragma unroll
        for (int j = 0; j < Shape::NI; ++j) {
            const int n = n0 + at.col + 16 * j;
            if (n >= a.dim)
                continue;
            const int64_t to = (int64_t(piece.first) + m) * stride + n;
            float v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r] * scale;
            const bool whole = vector && n + 4 <= a.dim;
            if (BF16) {
                uint16_t *out = (uint16_t *)grad_table + to;
                if (whole) {
                    if (ADD) {
                        const ushort4 old = *(const ushort4 *)out;
                        v[0] += widen(old.x), v[1] += widen(old.y);
                        v[2] += widen(old.z), v[3] += widen(old.w);
                    }
                    *(ushort4 *)out = make_ushort4(to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]),
                                                   to_bf16(v[3]));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (n + r < a.dim)
                            out[r] = to_bf16(ADD ? v[r] + widen(out[r]) : v[r]);
                }
            } else {
                float *out = (float *)grad_table + to;
                if (whole) {
                    float4 w = make_float4(v[0], v[1], v[2], v[3]);
                    if (ADD) {
                        const float4 old = *(const float4 *)out;
                        w.x += old.x, w.y += old.y, w.z += old.z, w.w += old.w;
                    }
                    *(float4 *)out = w;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (n + r < a.dim)
                            out[r] = ADD ? v[r] + out[r] : v[r];
                }
            }
        }
    }
}

template <class F>
hipError_t with_shape(int shape, F f) {
    switch (shape) {
    case kXentTiny: f(Tiny{}); break;
    case kXentSmall: f(Small{}); break;
    case kXentLarge: f(Large{}); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

int64_t tiles(int64_t rows, int64_t cols, int shape) {
    const int64_t t = xent_tile(shape);
    return (rows + t - 1) / t * ((cols + t - 1) / t);
}

}  // namespace

hipError_t launch_xent_pack(const XentPack &args, hipStream_t stream) {
    // one workgroup at least: it writes the count
    const int blocks = args.tokens ? tiles_of(args.tokens, kPackTokens * args.rounds) : 1;
    xent_pack_kernel<<<blocks, 256, 0, stream>>>(args);
    return hipGetLastError();
}

hipError_t launch_xent_copy(const uint16_t *src, int64_t stride, uint16_t *dst, int32_t dim,
                            int32_t ld, int64_t rows, hipStream_t stream) {
    xent_copy_kernel<<<uint32_t((rows + 3) / 4), 256, 0, stream>>>(src, stride, dst, dim, ld, rows);
    return hipGetLastError();
}

hipError_t launch_xent_logits(const XentArgs &args, int shape, float2 *parts, float *at_target,
                              hipStream_t stream) {
    return with_shape(shape, [&](auto s) {
        using Shape = decltype(s);
        xent_logits_kernel<Shape>
            <<<grid_of(tiles(args.tokens, args.vocab, shape)), Shape::kThreads, 0, stream>>>(
                args, parts, at_target);
    });
}

hipError_t launch_xent_reduce(const XentArgs &args, int32_t n_parts, const float2 *parts,
                              const float *at_target, float *loss, float *lse, float *mean,
                              hipStream_t stream) {
    xent_reduce_kernel<<<tiles_of(args.tokens, kReduceTokens), 256, 0, stream>>>(
        args, n_parts, parts, at_target, loss, lse, mean);
    return hipGetLastError();
}

hipError_t launch_xent_mean(const float *loss, int32_t tokens, const int32_t *kept, float *mean,
                            hipStream_t stream) {
    xent_mean_kernel<<<1, 1024, 0, stream>>>(loss, tokens, kept, mean);
    return hipGetLastError();
}

hipError_t launch_xent_probs(const XentArgs &args, int shape, const XentPiece &piece,
                             const float *lse, hipStream_t stream) {
    return with_shape(shape, [&](auto s) {
        using Shape = decltype(s);
        auto kernel = piece.low ? xent_probs_kernel<Shape, true> : xent_probs_kernel<Shape, false>;
        kernel<<<uint32_t(tiles(args.tokens, piece.ld, shape)), Shape::kThreads, 0, stream>>>(
            args, piece, lse);
    });
}

hipError_t launch_xent_hidden(const XentArgs &args, int shape, const XentPiece &piece,
                              int32_t splits, bool add, float *partial, hipStream_t stream) {
    return with_shape(shape, [&](auto s) {
        using Shape = decltype(s);
        xent_hidden_kernel<Shape>
            <<<uint32_t(tiles(args.tokens, args.dim, shape) * splits), Shape::kThreads, 0,
               stream>>>(args, piece, splits, add, partial);
    });
}

hipError_t launch_xent_hidden_out(const XentArgs &args, int32_t splits, const float *partial,
                                  const float *grad_loss, float grad_scale, bool mean,
                                  uint16_t *grad_hidden, int64_t stride, hipStream_t stream) {
    const int64_t blocks = int64_t(tiles_of(args.dim, 1024)) * args.tokens;
    xent_hidden_out_kernel<<<grid_of(blocks), 256, 0, stream>>>(
        args, splits, partial, grad_loss, grad_scale, mean, grad_hidden, stride);
    return hipGetLastError();
}

hipError_t launch_xent_table(const XentArgs &args, int shape, const XentPiece &piece,
                             const float *grad_loss, float grad_scale, bool mean, bool bf16_out,
                             bool add, void *grad_table, int64_t stride, float *partial,
                             hipStream_t stream) {
    const int64_t size = bf16_out ? 2 : 4;
    const bool vector = stride * size % 16 == 0 && (uintptr_t(grad_table) & 15) == 0;
    return with_shape(shape, [&](auto s) {
        using Shape = decltype(s);
        auto kernel = bf16_out ? (add ? xent_table_kernel<Shape, true, true>
                                      : xent_table_kernel<Shape, true, false>)
                               : (add ? xent_table_kernel<Shape, false, true>
                                      : xent_table_kernel<Shape, false, false>);
        kernel<<<uint32_t(tiles(piece.count, args.dim, shape)), Shape::kThreads, 0, stream>>>(
            args, piece, grad_loss, grad_scale, mean, grad_table, stride, vector, partial);
    });
}

}  // namespace lamb_mi355x
