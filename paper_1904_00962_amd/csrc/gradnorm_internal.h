// Layout shared by the kernels of the gradients' norms and clipping (gradnorm_kernels.hip)
// and their host side (gradnorm_api.cpp). Not installed; the public interface is
// include/lamb_ops.h.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace lamb_mi355x {

// One tensor of a plan's list. Its elements are worked on by `chunks` workgroups.
struct GradTensor {
    const void *in;
    void *out;  // NULL in plans that only take norms
    int64_t numel;
    int32_t in_bf16, out_bf16;
    int32_t first_chunk, chunks;
};

struct GradList {
    const GradTensor *tensors;
    const int32_t *chunk_tensor;  // the tensor of each chunk
    int32_t n, chunks;
    int32_t chunk;  // elements of one, a multiple of kGradStep
    int32_t norm;   // a lamb_norm
    double *partials;  // [chunks]
    double *powers;    // [n]: sums of squares or magnitudes, or the largest magnitude
};

constexpr int kGradBlock = 256;
constexpr int kGradStep = kGradBlock * 8;  // elements that a workgroup loads at once

hipError_t launch_grad_norms(const GradList &list, hipStream_t stream);
hipError_t launch_grad_totals(const GradList &list, double *norms, double *total,
                              hipStream_t stream);
// out = scale min(1, max_norm / (|scale| total)) in, or scale in where total is not finite.
hipError_t launch_grad_clip(const GradList &list, const double *total, double max_norm,
                            double scale, int32_t *nonfinite_out, hipStream_t stream);

}  // namespace lamb_mi355x
