// Layout shared by the kernels of the Newton-Schulz products (ortho_kernels.hip)
// and their host side (ortho_api.cpp). Not installed; the public interface is
// include/lamb_ops.h.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace lamb_mi355x {

// X, A and P are held as 16-bit floats times kNsScale. Their entries are at most
// their largest singular value, which the host keeps under kNsLargest for P and
// kNsLargestX for X, so kNsScale times that stays below the format's 65504; and
// an entry of 2^-14, about the smallest of a 16384 x 16384 matrix, is still a normal
// number with a normal low part.
constexpr float kNsScale = 8192.0f;
constexpr double kNsLargest = 7.75, kNsLargestX = 2.75;

// Elements per workgroup of the elementwise passes, in units of 8 columns.
constexpr int kNsBlock = 256;
constexpr int kNsUnits = 4;  // units per thread
constexpr int kNsBlockUnits = kNsBlock * kNsUnits;

// One matrix. `tall`: rows > cols, and A = X^T X, X <- X P; else A = X X^T, X <- P X.
struct NsMatrix {
    const void *in;     // orthogonalize: the input; Muon: the gradient
    void *out;          // orthogonalize: the output; Muon: the parameters x
    float *m;           // Muon: the momentum
    uint16_t *x[2];     // X of even and odd iterations, [rows][ld]; low parts x_low further
    uint16_t *gram[2];  // A, [side][side_ld]; low parts gram_low further
    uint16_t *poly[2];  // P, likewise, and with `chain` also ...
    uint16_t *q, *t;    // Q and T of a chain, likewise (see ns_chain)
    int64_t in_stride, out_stride;
    int64_t x_low, gram_low;
    int32_t rows, cols, ld, side, side_ld, tall;
    int32_t first_block, blocks;  // its workgroups of the elementwise passes
    int32_t vector;               // rows of in, out and m allow 16-byte accesses
    int32_t wd;                   // Muon: decay applies
    int32_t chain;                // iterations in chains
    int32_t reserved;
};
static_assert(sizeof(NsMatrix) == 168, "NsMatrix layout");

// One tile of a product.
struct NsTile {
    int32_t matrix;
    int32_t row, col;  // in tiles
    int32_t product;   // an NsProduct, for launch_ns_product
};

// Chains. As every P is a polynomial of A, all of them commute, and n iterations can be
// taken on the short side alone: with A_0 = X X^T,
//   P_i = a I + b A_i + c A_i^2,  T = P_i A_i,  A_{i+1} = T P_i,  Q_i = P_i Q_{i-1},
// and at the end X <- Q X. For a matrix of L x S this costs 3 S^3 (symmetric halves) an
// iteration beside S^3 for Q, in place of 3 L S^2. The rounding of A hides singular
// values below its square root, and n iterations multiply what it hides by up to
// 3.4^(2 n): chains are kept to kNsChainSplit and kNsChainHalf iterations, which leave
// the result as exact as direct iterations do (256 x 1024 matrices of rank 32 and 1e-2 of
// noise: 6.9e-6 and 1.7e-2 off, 9.7e-6 and 2.1e-2 directly; rank 1 and 1e-4: 6.6e-5 and
// 1.4e-1, 5.9e-5 and 1.5e-1. Five at once ended some 30 times as far off).
constexpr int32_t kNsChainSplit = 3, kNsChainHalf = 2;
// Q is held times kNsQScale: its entries reach those of P to the third power.
constexpr float kNsQScale = 128.0f;
enum NsProduct : int32_t { kNsQ = 0, kNsT = 1, kNsA = 2 };
// Where iteration `turn` of a chain finds A and P is [turn & 1]; Q is P at first, then
// q, then the P before.

// Tile shapes of the products, all square.
enum NsShape : int32_t { kNsTiny = 0, kNsSmall = 1, kNsLarge = 2 };
constexpr int32_t ns_tile(int32_t shape) { return 64 << shape; }

enum NsKind : int32_t { kNsBf16Out = 0, kNsF32Out = 1, kNsMuon = 2 };

struct NsStep {
    float a, b, c;
    float eps;
    // Muon
    double momentum, from_grad;  // m <- momentum m + from_grad g
    float decay;                 // x <- decay x - lr s O (decay 1 where the mask is off)
    float lr;
    int32_t nesterov;
    int32_t scale;               // a lamb_muon_scale
};

// Elementwise passes over `blocks` workgroups (block_matrix: each one's matrix).
// `flag` non-null: a skip_nonfinite step. The check raises flag[0], the norm pass
// obeys it and copies it to flag[1], which the last update obeys, and the convert
// pass clears it for the next step; nothing depends on a host counter.
hipError_t launch_ns_check(const NsMatrix *matrices, const int32_t *block_matrix, int32_t blocks,
                           bool bf16_in, float grad_scale, uint32_t *flag, hipStream_t stream);
hipError_t launch_ns_norms(const NsMatrix *matrices, const int32_t *block_matrix, int32_t blocks,
                           bool muon, bool bf16_in, const NsStep &step, double *partials,
                           uint32_t *flag, int32_t *nonfinite_out, hipStream_t stream);
hipError_t launch_ns_convert(const NsMatrix *matrices, const int32_t *block_matrix,
                             int32_t blocks, bool muon, bool bf16_in, bool split,
                             const NsStep &step, const double *partials, uint32_t *flag,
                             hipStream_t stream);
// Products over `n` tiles of shape `shape`. `turn`: the iteration of matrices with
// `chain` in their chain. `parity`: which X is read, [0] of matrices without a chain,
// [1] of those with one.
struct NsTurn {
    int32_t turn;
    int32_t parity[2];
};
hipError_t launch_ns_gram(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                          bool split, const NsTurn &turn, hipStream_t stream);
hipError_t launch_ns_poly(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                          bool split, const NsTurn &turn, const NsStep &step, hipStream_t stream);
// The products of a chain, each tile's by its `product`.
hipError_t launch_ns_product(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                             bool split, const NsTurn &turn, hipStream_t stream);
// `last`: the result goes to `out` as `kind` says, else to the other X.
hipError_t launch_ns_update(const NsMatrix *matrices, const NsTile *tiles, int32_t n, int shape,
                            bool split, const NsTurn &turn, bool last, NsKind kind,
                            const NsStep &step, const uint32_t *flag, hipStream_t stream);

}  // namespace lamb_mi355x
