// Layout shared by the kernels of the token table (embed_kernels.hip) and their host
// side (embed_api.cpp). Not installed; the public interface is include/lamb_ops.h.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace lamb_mi355x {

struct EmbedArgs {
    const void *ids;
    int32_t wide;  // ids are 64-bit
    int64_t tokens, vocab;
    int32_t dim;
    float scale;
};

// out[i] = scale table[ids[i]]; NaN where the id is outside the table.
struct EmbedRows {
    const void *table;
    void *out;
    int64_t table_stride, out_stride;
    int32_t table_bf16, out_bf16;
    int32_t vector;  // rows of both are 16-byte aligned
};
hipError_t launch_embed(const EmbedArgs &args, const EmbedRows &rows, hipStream_t stream);

// Sorting: a workgroup of kSortWaves waves takes the ids of one range of the
// vocabulary out of all tokens.
constexpr int kSortWaves = 16;
constexpr int32_t kSortIds = 128;    // ids of a range where tokens are few
constexpr int32_t kSortIdsMost = 512;
constexpr int32_t sort_ids(int64_t tokens) {
    // Every workgroup reads every id, so many tokens are given fewer, wider ranges.
    return tokens <= 32768 ? kSortIds : tokens <= 262144 ? 2 * kSortIds : kSortIdsMost;
}

// Summing: a wave takes kSumTokens tokens of the sorted order and kSumColumns columns,
// or kZeroRows rows of the table that no token names.
constexpr int32_t kSumTokens = 16;
constexpr int32_t kZeroRows = 8;
constexpr int32_t kSumColumns = 512;
// Joining: chunks' sums that are added up by themselves, before they join the others, so
// that a chain of fp32 sums stays short: 2^20 like rows of one id end 6e-4 off in one chain.
constexpr int64_t kJoinChunks = 64;

// order[0 .. first[vocab]): the tokens in the order of their ids, those of one id in
// theirs; first[v]: where id v's tokens begin. Ids outside the table and `skip` are
// left out.
hipError_t launch_embed_sort(const EmbedArgs &args, int64_t skip, int32_t *order, int32_t *sorted,
                             int32_t *first, hipStream_t stream);

struct EmbedGrad {
    const void *rows;  // gradients of the looked-up rows
    void *table;       // gradient of the table
    int64_t rows_stride, table_stride;
    int32_t rows_bf16, table_bf16;
    int32_t add;
    int32_t vector;
    const int32_t *order, *sorted, *first;
    float *partial;  // [2 * chunks][columns]: sums of ids that do not begin or end in a chunk
    int32_t columns;  // dim, rounded up to kSumColumns
};
hipError_t launch_embed_sum(const EmbedArgs &args, const EmbedGrad &grad, hipStream_t stream);
hipError_t launch_embed_join(const EmbedArgs &args, const EmbedGrad &grad, hipStream_t stream);

}  // namespace lamb_mi355x
