// Host side of the root-mean-square norm's entry points of include/lamb_ops.h.
#include <math.h>

#include "ops_host.h"
#include "rms_internal.h"

using namespace lamb_mi355x;

namespace {

lamb_status check_rows(const char *what, const void *p, int64_t rows, int64_t stride, int64_t dim,
                       int64_t size) {
    if (rows && !p)
        return fail(LAMB_ENULL, "%s must not be NULL", what);
    if (stride < dim || stride > kMaxStride)
        return fail(LAMB_EINVAL, "%s: the row stride is below dim, or above 2^36", what);
    if (!aligned_to(p, uintptr_t(size)))
        return fail(LAMB_EALIGN, "%s is not aligned to its elements", what);
    return LAMB_OK;
}

lamb_status check_type(const char *what, int32_t dtype) {
    return is_float(dtype) ? LAMB_OK : fail(LAMB_EINVAL, "%s is float32 or bfloat16", what);
}

lamb_status check(const lamb_rms *r) {
    if (!r)
        return fail(LAMB_ENULL, "rms must not be NULL");
    if (r->tokens < 0 || r->tokens > kMaxTokens || r->dim < 1 || r->dim > kMaxDim)
        return fail(LAMB_EINVAL, "tokens %lld, dim %lld: need 0 to 2^24, 1 to 2^16",
                    (long long)r->tokens, (long long)r->dim);
    if (!std::isfinite(r->eps) || r->eps < 0.0f)
        return fail(LAMB_EINVAL, "eps = %g, need finite and >= 0", double(r->eps));
    lamb_status st = check_type("x", r->x_dtype);
    if (st == LAMB_OK)
        st = check_rows("x", r->x, r->tokens, r->x_stride, r->dim, size_of(r->x_dtype));
    if (st == LAMB_OK && r->residual) {
        st = check_type("residual", r->residual_dtype);
        if (st == LAMB_OK && r->x_dtype == LAMB_DTYPE_F32 && r->residual_dtype != LAMB_DTYPE_F32)
            st = fail(LAMB_EINVAL, "the residual of a float32 x is float32");
        if (st == LAMB_OK)
            st = check_rows("residual", r->residual, r->tokens, r->residual_stride, r->dim,
                            size_of(r->residual_dtype));
    }
    if (st == LAMB_OK && r->weight) {
        st = check_type("weight", r->weight_dtype);
        if (st == LAMB_OK && !aligned_to(r->weight, uintptr_t(size_of(r->weight_dtype))))
            st = fail(LAMB_EALIGN, "weight is not aligned to its elements");
    }
    return st;
}

RmsArgs args_of(const lamb_rms &r) {
    return RmsArgs{r.x,
                   r.residual,
                   r.weight,
                   r.x_stride,
                   r.residual_stride,
                   r.tokens,
                   int32_t(r.dim),
                   r.x_dtype == LAMB_DTYPE_BF16,
                   r.residual_dtype == LAMB_DTYPE_BF16,
                   r.weight_dtype == LAMB_DTYPE_BF16,
                   r.eps,
                   1.0 / double(r.dim)};
}

// What a call touches, up to eight pieces of it.
struct Spans {
    Span list[8];
    size_t n = 0;
    const lamb_rms &r;

    explicit Spans(const lamb_rms &rms) : r(rms) {
        if (r.weight)
            list[n++] = span_of(r.weight, uint64_t(r.dim * size_of(r.weight_dtype)), false, 0,
                                "weight");
    }
    void rows(const void *p, int64_t stride, int64_t size, bool written, const char *what) {
        list[n++] = span_of_rows(p, r.tokens, stride, r.dim, size, written, 0, what);
    }
    // An operand that `to` overwrites in place (its address, stride and size) does not
    // overlap it: a lane writes the elements that it read itself.
    void read(const void *p, int64_t stride, int64_t size, const void *to, int64_t to_stride,
              int64_t to_size, const char *what) {
        const bool in_place = p == to && stride == to_stride && size == to_size;
        if (p && !in_place)
            rows(p, stride, size, false, what);
    }
    lamb_status check() { return check_spans(list, n); }
};

lamb_status forward(const lamb_rms *rms, void *summed, int64_t summed_stride, void *out,
                    int64_t out_stride, int64_t out_size, int32_t out_bf16, float *scales,
                    int32_t group, void *stream) {
    const lamb_rms &r = *rms;
    lamb_status st = check_rows("out", out, r.tokens, out_stride, r.dim, out_size);
    const int64_t sum_size = size_of(r.residual_dtype);
    if (st == LAMB_OK && summed) {
        if (!r.residual)
            return fail(LAMB_EINVAL, "summed needs a residual");
        st = check_rows("summed", summed, r.tokens, summed_stride, r.dim, sum_size);
    }
    if (st != LAMB_OK)
        return st;
    const int64_t groups = group ? (r.dim + group - 1) / group : 1;
    Spans spans(r);
    const void *const written[2] = {out, summed};
    const int64_t strides[2] = {out_stride, summed_stride}, sizes[2] = {out_size, sum_size};
    auto reads = [&](const void *p, int64_t stride, int64_t size, const char *what) {
        // in place of either result
        const int k = p == out && !scales ? 0 : 1;
        spans.read(p, stride, size, written[k], strides[k], sizes[k], what);
    };
    reads(r.x, r.x_stride, size_of(r.x_dtype), "x");
    reads(r.residual, r.residual_stride, sum_size, "residual");
    spans.rows(out, out_stride, out_size, true, "out");
    if (summed)
        spans.rows(summed, summed_stride, sum_size, true, "summed");
    if (scales)
        spans.list[spans.n++] =
            span_of(scales, uint64_t(r.tokens * groups * 4), true, 0, "scales");
    st = spans.check();
    if (st != LAMB_OK || r.tokens == 0)
        return st;
    const RmsOut o{summed,   out,    summed_stride, out_stride,
                   out_bf16, scales, group,         int32_t(groups)};
    const hipError_t err = launch_rms(args_of(r), o, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

struct Layout {
    int64_t columns;
    size_t stats, bytes;
};

Layout layout_of(const lamb_rms &r) {
    Layout l{};
    l.columns = round_up(r.dim, 8);
    const int64_t partials = rms_most_partials(r.tokens, int32_t(r.dim));
    l.stats = size_t(round_up(partials * l.columns * 4, 256));
    l.bytes = l.stats + (r.dim > kRmsHeldDim ? size_t(round_up(r.tokens * 16, 256)) : 0);
    return l;
}

}  // namespace

extern "C" {

lamb_status lamb_rms_forward(const lamb_rms *rms, void *summed, int64_t summed_stride, void *out,
                             int64_t out_stride, int32_t out_dtype, void *stream) {
    lamb_status st = check(rms);
    if (st == LAMB_OK)
        st = check_type("out", out_dtype);
    if (st != LAMB_OK)
        return st;
    return forward(rms, summed, summed_stride, out, out_stride, size_of(out_dtype),
                   out_dtype == LAMB_DTYPE_BF16, nullptr, 0, stream);
}

lamb_status lamb_rms_quantize(const lamb_rms *rms, void *summed, int64_t summed_stride, void *out,
                              int64_t out_stride, float *scales, int32_t group, void *stream) {
    const lamb_status st = check(rms);
    if (st != LAMB_OK)
        return st;
    if (group != 0 && group != 32 && group != 64 && group != 128 && group != 256)
        return fail(LAMB_EINVAL, "group = %d, need 0 (a row), 32, 64, 128 or 256", group);
    if (rms->tokens && !scales)
        return fail(LAMB_ENULL, "scales must not be NULL");
    if (!aligned_to(scales, 4))
        return fail(LAMB_EALIGN, "scales are not aligned to their elements");
    if (rms->tokens == 0)
        scales = nullptr;
    return forward(rms, summed, summed_stride, out, out_stride, 1, 0, scales, group, stream);
}

lamb_status lamb_rms_workspace(const lamb_rms *rms, size_t *bytes) {
    const lamb_status st = check(rms);
    if (st != LAMB_OK)
        return st;
    if (!bytes)
        return fail(LAMB_ENULL, "bytes must not be NULL");
    *bytes = layout_of(*rms).bytes;
    return LAMB_OK;
}

lamb_status lamb_rms_backward(const lamb_rms *rms, const lamb_rms_grads *grads, void *workspace,
                              size_t workspace_bytes, void *stream_in) {
    lamb_status st = check(rms);
    if (st != LAMB_OK)
        return st;
    if (!grads)
        return fail(LAMB_ENULL, "grads must not be NULL");
    const lamb_rms &r = *rms;
    const lamb_rms_grads &g = *grads;
    if (r.residual)
        return fail(LAMB_EINVAL, "the gradients are of the sum: residual must be NULL, x the sum");
    if (g.add_weight & ~1)
        return fail(LAMB_EINVAL, "grads.add_weight must be 0 or 1");
    if (g.reserved != 0)
        return fail(LAMB_EINVAL, "grads.reserved must be 0");
    st = check_type("grad_out", g.grad_out_dtype);
    if (st == LAMB_OK)
        st = check_rows("grad_out", g.grad_out, r.tokens, g.grad_out_stride, r.dim,
                        size_of(g.grad_out_dtype));
    if (st == LAMB_OK && (g.grad_x || g.grad_sum))
        st = check_type("grad_x", g.grad_x_dtype);
    const int64_t dx_size = size_of(g.grad_x_dtype);
    if (st == LAMB_OK && g.grad_x)
        st = check_rows("grad_x", g.grad_x, r.tokens, g.grad_x_stride, r.dim, dx_size);
    if (st == LAMB_OK && g.grad_sum)
        st = check_rows("grad_sum", g.grad_sum, r.tokens, g.grad_sum_stride, r.dim, dx_size);
    if (st == LAMB_OK && g.grad_weight) {
        st = check_type("grad_weight", g.grad_weight_dtype);
        if (st == LAMB_OK && !aligned_to(g.grad_weight, uintptr_t(size_of(g.grad_weight_dtype))))
            st = fail(LAMB_EALIGN, "grad_weight is not aligned to its elements");
    }
    if (st != LAMB_OK)
        return st;
    const Layout l = layout_of(r);
    // only these need it
    const bool held = g.grad_weight || r.dim > kRmsHeldDim;
    if (held && r.tokens) {
        st = check_workspace(workspace, workspace_bytes, l.bytes);
        if (st != LAMB_OK)
            return st;
    }
    Spans spans(r);
    auto reads = [&](const void *p, int64_t stride, int64_t size, const char *what) {
        spans.read(p, stride, size, g.grad_x, g.grad_x_stride, dx_size, what);
    };
    reads(r.x, r.x_stride, size_of(r.x_dtype), "x");
    reads(g.grad_out, g.grad_out_stride, size_of(g.grad_out_dtype), "grad_out");
    reads(g.grad_sum, g.grad_sum_stride, dx_size, "grad_sum");
    if (g.grad_x)
        spans.rows(g.grad_x, g.grad_x_stride, dx_size, true, "grad_x");
    if (g.grad_weight)
        spans.list[spans.n++] =
            span_of(g.grad_weight, uint64_t(r.dim * size_of(g.grad_weight_dtype)), true, 0,
                    "grad_weight");
    if (held && r.tokens)
        spans.list[spans.n++] = span_of(workspace, l.bytes, true, 0, "workspace");
    st = spans.check();
    if (st != LAMB_OK || (!g.grad_x && !g.grad_weight))
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    const RmsArgs args = args_of(r);
    char *work = static_cast<char *>(workspace);
    RmsGrad grad{g.grad_out,
                 g.grad_sum,
                 g.grad_x,
                 g.grad_weight,
                 g.grad_out_stride,
                 g.grad_sum_stride,
                 g.grad_x_stride,
                 g.grad_out_dtype == LAMB_DTYPE_BF16,
                 g.grad_x_dtype == LAMB_DTYPE_BF16,
                 g.grad_weight_dtype == LAMB_DTYPE_BF16,
                 g.add_weight,
                 reinterpret_cast<float *>(work),
                 0,
                 int32_t(l.columns),
                 reinterpret_cast<double *>(work + l.stats)};
    grad.partials = rms_partials(args, grad);
    hipError_t err = hipSuccess;
    if (r.tokens)
        err = launch_rms_grad(args, grad, stream);
    if (err == hipSuccess && g.grad_weight && (r.tokens || !g.add_weight))
        err = launch_rms_join(args, grad, stream);
    return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
}

}  // extern "C"
