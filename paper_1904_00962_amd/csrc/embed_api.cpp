// Host side of the token table's entry points of include/lamb_ops.h.
#include <math.h>

#include "embed_internal.h"
#include "ops_host.h"

using namespace lamb_mi355x;

namespace {

lamb_status check(const lamb_embed *e) {
    if (!e)
        return fail(LAMB_ENULL, "embed must not be NULL");
    if (e->tokens < 0 || e->tokens > kMaxTokens || e->vocab < 1 || e->vocab > kMaxVocab ||
        e->dim < 1 || e->dim > kMaxDim)
        return fail(LAMB_EINVAL,
                    "tokens %lld, vocab %lld, dim %lld: need 0 to 2^24, 1 to 2^24, 1 to 2^16",
                    (long long)e->tokens, (long long)e->vocab, (long long)e->dim);
    if (!is_id(e->id_dtype))
        return fail(LAMB_EINVAL, "ids are int32 or int64");
    if (!std::isfinite(e->scale))
        return fail(LAMB_EINVAL, "scale = %g must be finite", double(e->scale));
    if (e->tokens && !e->ids)
        return fail(LAMB_ENULL, "ids must not be NULL");
    if (!aligned_to(e->ids, uintptr_t(size_of(e->id_dtype))))
        return fail(LAMB_EALIGN, "ids are not aligned to their elements");
    return LAMB_OK;
}

lamb_status check_matrix(const char *what, const void *p, int64_t rows, int64_t stride,
                         int64_t dim, int32_t dtype) {
    if (!is_float(dtype))
        return fail(LAMB_EINVAL, "%s is float32 or bfloat16", what);
    if (rows && !p)
        return fail(LAMB_ENULL, "%s must not be NULL", what);
    if (stride < dim || stride > kMaxStride)
        return fail(LAMB_EINVAL, "%s: the row stride is below dim, or above 2^36", what);
    if (!aligned_to(p, uintptr_t(size_of(dtype))))
        return fail(LAMB_EALIGN, "%s is not aligned to its elements", what);
    return LAMB_OK;
}

bool whole_rows(const void *p, int64_t stride, int32_t dtype) {
    return aligned_to(p, 16) && stride * size_of(dtype) % 16 == 0;
}

EmbedArgs args_of(const lamb_embed &e) {
    return EmbedArgs{e.ids, e.id_dtype == LAMB_DTYPE_I64, e.tokens, e.vocab, int32_t(e.dim),
                     e.scale};
}

struct Layout {
    int64_t columns;
    size_t order, sorted, first, partial, bytes;
};

Layout layout_of(const lamb_embed &e) {
    Layout l{};
    l.columns = round_up(e.dim, kSumColumns);
    const int64_t chunks = (e.tokens + kSumTokens - 1) / kSumTokens;
    auto take = [&](int64_t bytes) {
        const size_t at = l.bytes;
        l.bytes += size_t(round_up(bytes, 256));
        return at;
    };
    l.order = take(4 * e.tokens);
    l.sorted = take(4 * e.tokens);
    l.first = take(4 * (e.vocab + 1));
    l.partial = take(2 * chunks * l.columns * 4);
    return l;
}

}  // namespace

extern "C" {

lamb_status lamb_embed_forward(const lamb_embed *embed, const void *table, int64_t table_stride,
                               int32_t table_dtype, void *out, int64_t out_stride,
                               int32_t out_dtype, void *stream) {
    lamb_status st = check(embed);
    if (st != LAMB_OK)
        return st;
    const lamb_embed &e = *embed;
    st = check_matrix("table", table, e.vocab, table_stride, e.dim, table_dtype);
    if (st == LAMB_OK)
        st = check_matrix("out", out, e.tokens, out_stride, e.dim, out_dtype);
    if (st != LAMB_OK)
        return st;
    Span spans[] = {
        span_of(e.ids, uint64_t(e.tokens * size_of(e.id_dtype)), false, 0, "ids"),
        span_of_rows(table, e.vocab, table_stride, e.dim, size_of(table_dtype), false, 0, "table"),
        span_of_rows(out, e.tokens, out_stride, e.dim, size_of(out_dtype), true, 0, "out")};
    st = check_spans(spans, sizeof spans / sizeof spans[0]);
    if (st != LAMB_OK || e.tokens == 0)
        return st;
    const EmbedRows rows{table,
                         out,
                         table_stride,
                         out_stride,
                         table_dtype == LAMB_DTYPE_BF16,
                         out_dtype == LAMB_DTYPE_BF16,
                         whole_rows(table, table_stride, table_dtype) &&
                             whole_rows(out, out_stride, out_dtype)};
    const hipError_t err = launch_embed(args_of(e), rows, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

lamb_status lamb_embed_workspace(const lamb_embed *embed, size_t *bytes) {
    const lamb_status st = check(embed);
    if (st != LAMB_OK)
        return st;
    if (!bytes)
        return fail(LAMB_ENULL, "bytes must not be NULL");
    *bytes = layout_of(*embed).bytes;
    return LAMB_OK;
}

lamb_status lamb_embed_backward(const lamb_embed *embed, const void *grad_out,
                                int64_t grad_out_stride, int32_t grad_out_dtype, void *grad_table,
                                int64_t grad_table_stride, int32_t grad_table_dtype,
                                int64_t padding_id, int32_t add, void *workspace,
                                size_t workspace_bytes, void *stream_in) {
    lamb_status st = check(embed);
    if (st != LAMB_OK)
        return st;
    const lamb_embed &e = *embed;
    if (add & ~1)
        return fail(LAMB_EINVAL, "add must be 0 or 1");
    st = check_matrix("grad_out", grad_out, e.tokens, grad_out_stride, e.dim, grad_out_dtype);
    if (st == LAMB_OK)
        st = check_matrix("grad_table", grad_table, e.vocab, grad_table_stride, e.dim,
                          grad_table_dtype);
    if (st != LAMB_OK)
        return st;
    const Layout l = layout_of(e);
    st = check_workspace(workspace, workspace_bytes, l.bytes);
    if (st != LAMB_OK)
        return st;
    Span spans[] = {
        span_of(e.ids, uint64_t(e.tokens * size_of(e.id_dtype)), false, 0, "ids"),
        span_of_rows(grad_out, e.tokens, grad_out_stride, e.dim, size_of(grad_out_dtype), false, 0,
                     "grad_out"),
        span_of_rows(grad_table, e.vocab, grad_table_stride, e.dim, size_of(grad_table_dtype), true,
                     0, "grad_table"),
        span_of(workspace, l.bytes, true, 0, "workspace")};
    st = check_spans(spans, sizeof spans / sizeof spans[0]);
    if (st != LAMB_OK || (e.tokens == 0 && add))
        return st;
    char *work = static_cast<char *>(workspace);
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    const EmbedArgs args = args_of(e);
    int32_t *order = reinterpret_cast<int32_t *>(work + l.order);
    int32_t *sorted = reinterpret_cast<int32_t *>(work + l.sorted);
    int32_t *first = reinterpret_cast<int32_t *>(work + l.first);
    const EmbedGrad grad{grad_out,
                         grad_table,
                         grad_out_stride,
                         grad_table_stride,
                         grad_out_dtype == LAMB_DTYPE_BF16,
                         grad_table_dtype == LAMB_DTYPE_BF16,
                         add,
                         whole_rows(grad_out, grad_out_stride, grad_out_dtype) &&
                             whole_rows(grad_table, grad_table_stride, grad_table_dtype),
                         order,
                         sorted,
                         first,
                         reinterpret_cast<float *>(work + l.partial),
                         int32_t(l.columns)};
    hipError_t err = launch_embed_sort(args, padding_id, order, sorted, first, stream);
    if (err == hipSuccess)
        err = launch_embed_sum(args, grad, stream);
    if (err == hipSuccess && e.tokens > kSumTokens)  // else one chunk holds every id
        err = launch_embed_join(args, grad, stream);
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

}  // extern "C"
