// Layout shared by the kernels of the cross entropy (xent_kernels.hip) and their
// host side (xent_api.cpp). Not installed; the public interface is
// include/lamb_ops.h.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace lamb_mi355x {

// Tile shapes, all square.
enum XentShape : int32_t { kXentTiny = 0, kXentSmall = 1, kXentLarge = 2 };
constexpr int32_t xent_tile(int32_t shape) { return 64 << shape; }

// Tokens that a workgroup of the packing pass takes at once, and how often it does. Each
// counts the tokens before its own first, so there are at most 1024 workgroups, four to a
// CU: the work of counting then grows as the tokens do. A call of 2^20 tokens and 64
// columns against 64 words takes 1.0 ms so, 14.8 with one group to a workgroup; of 65536
// 72 and 113 us.
constexpr int kPackTokens = 16;
constexpr int32_t pack_rounds(int64_t tokens) {
    return tokens > 1024 * kPackTokens
               ? int32_t((tokens + 1024 * kPackTokens - 1) / (1024 * kPackTokens))
               : 1;
}
// Tokens that one chain of fp32 sums takes: a matrix instruction rounds each product to the
// sum's last place, which costs a column of equal values (0.7 times the same probability)
// 5e-5 after 65536 tokens, 7e-4 after 2^20 and 8e-3 after 2^22. More tokens are summed in
// chains of this many, which add up in memory.
constexpr int32_t kChainTokens = 32768;
constexpr int kReduceTokens = 16;  // tokens per workgroup of the logsumexp pass

// What every pass of a call reads. `hidden` is the packed copy of the tokens that
// count, rows `ld` apart with zeros from dim to ld; `table` the caller's, or a copy
// laid out likewise.
struct XentArgs {
    const uint16_t *hidden;
    const uint16_t *table;
    int64_t ld, table_ld;
    int32_t dim, vocab, tokens;
    const int32_t *kept;    // tokens that count
    const int32_t *source;  // packed row -> token
    const int32_t *target;  // packed row -> target, -1 where it is outside the vocabulary
};

struct XentPack {
    const uint16_t *hidden;
    int64_t stride;
    const void *targets;
    int32_t wide;  // targets are 64-bit
    int32_t vector;
    int64_t ignore;
    int32_t dim, ld, vocab, tokens;
    int32_t rounds;
    uint16_t *packed;
    int32_t *kept, *source, *target;
    float *loss, *lse;           // forward: of the tokens that do not count, 0
    uint16_t *grad_hidden;       // backward: likewise, rows grad_stride apart
    int64_t grad_stride;
};

// Copies the rows of the tokens that count together, in their order.
hipError_t launch_xent_pack(const XentPack &args, hipStream_t stream);
// dst[r][0 .. ld) = src[r][0 .. dim) and zeros, `rows` rows.
hipError_t launch_xent_copy(const uint16_t *src, int64_t stride, uint16_t *dst, int32_t dim,
                            int32_t ld, int64_t rows, hipStream_t stream);
// Logits of all of the vocabulary, tile by tile: each tile column's maxima and sums of
// exponentials, parts[column][token], and the targets' logits.
hipError_t launch_xent_logits(const XentArgs &args, int shape, float2 *parts, float *at_target,
                              hipStream_t stream);
// `mean` non-null: the mean too, where kReduceTokens hold all tokens.
hipError_t launch_xent_reduce(const XentArgs &args, int32_t n_parts, const float2 *parts,
                              const float *at_target, float *loss, float *lse, float *mean,
                              hipStream_t stream);
// mean = sum of the losses over the count of tokens (0 without any).
hipError_t launch_xent_mean(const float *loss, int32_t tokens, const int32_t *kept, float *mean,
                            hipStream_t stream);

// One piece of the vocabulary: rows [first, first + count) of the table; probs is
// [tokens][ld] with zeros from count to ld, and so is low, what the rounding of probs
// leaves, where the table's gradient is fp32 (else null).
struct XentPiece {
    int32_t first, count, ld;
    uint16_t *probs, *low;
};

// probs = softmax - one at the target, in bf16; low = the rest of it, in bf16 again.
hipError_t launch_xent_probs(const XentArgs &args, int shape, const XentPiece &piece,
                             const float *lse, hipStream_t stream);
// partial[split] (tokens x dim, fp32) = or += probs' share of the piece times the table.
hipError_t launch_xent_hidden(const XentArgs &args, int shape, const XentPiece &piece,
                              int32_t splits, bool add, float *partial, hipStream_t stream);
// The sum over the splits, scaled, to the tokens' rows of grad_hidden.
hipError_t launch_xent_hidden_out(const XentArgs &args, int32_t splits, const float *partial,
                                  const float *grad_loss, float grad_scale, bool mean,
                                  uint16_t *grad_hidden, int64_t stride, hipStream_t stream);
// grad_table's rows of the piece = (or +=) scale probs^T hidden; fp32: (probs + low)^T hidden.
// partial: [piece.count][ld] in fp32, for more than kChainTokens tokens.
hipError_t launch_xent_table(const XentArgs &args, int shape, const XentPiece &piece,
                             const float *grad_loss, float grad_scale, bool mean, bool bf16_out,
                             bool add, void *grad_table, int64_t stride, float *partial,
                             hipStream_t stream);

}  // namespace lamb_mi355x
