// Layout shared by the kernels of the root-mean-square norm (rms_kernels.hip) and their
// host side (rms_api.cpp). Not installed; the public interface is include/lamb_ops.h.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace lamb_mi355x {

constexpr int kRmsBlock = 256;  // threads of a workgroup, at least

struct RmsArgs {
    const void *x, *residual, *weight;  // residual, weight: may be NULL
    int64_t x_stride, residual_stride;
    int64_t tokens;
    int32_t dim;
    int32_t x_bf16, residual_bf16, weight_bf16;
    float eps;
    double per_column;  // 1 / dim
};

struct RmsOut {
    void *summed;  // of the residual's type; may be NULL
    void *out;     // e4m3 bytes where there are scales
    int64_t summed_stride, out_stride;
    int32_t out_bf16;
    float *scales;          // [tokens][groups], or NULL
    int32_t group, groups;  // columns that share a scale: a power of two, or 0 for a row
};
hipError_t launch_rms(const RmsArgs &args, const RmsOut &out, hipStream_t stream);

// Rows wider than this take two passes backward: a lane would have to hold more columns'
// sums than it has registers for.
constexpr int32_t kRmsHeldDim = 8192;
constexpr int32_t kRmsFoldRows = 32;  // rows whose terms of the weight's gradient are one sum
constexpr int32_t kRmsWideRows = 16;  // rows of a workgroup in the second pass of wide rows

struct RmsGrad {
    const void *grad_out, *grad_sum;  // grad_sum: may be NULL
    void *grad_x, *grad_weight;       // either may be NULL
    int64_t grad_out_stride, grad_sum_stride, grad_x_stride;
    int32_t grad_out_bf16, grad_x_bf16, grad_weight_bf16;  // grad_sum is as grad_x
    int32_t add_weight;
    float *partial;     // [partials][columns]: parts of the weight's gradient
    int64_t partials;   // rows of it
    int32_t columns;    // dim, rounded up to 8
    double *stats;      // [tokens][2], for wide rows: 1 / rms, and the mean of g x / rms
};
// Rows of RmsGrad::partial in a call, and in any of these sizes.
int64_t rms_partials(const RmsArgs &args, const RmsGrad &grad);
int64_t rms_most_partials(int64_t tokens, int32_t dim);
hipError_t launch_rms_grad(const RmsArgs &args, const RmsGrad &grad, hipStream_t stream);
hipError_t launch_rms_join(const RmsArgs &args, const RmsGrad &grad, hipStream_t stream);

}  // namespace lamb_mi355x
