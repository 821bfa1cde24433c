// Layout shared by the kernels of the gradients' norms and clipping (gradnorm_kernels.hip)
// and their host side (gradnorm_api.cpp). Not installed; the public interface is
// include/lamb_ops.h.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace lamb_mi355x {

// One tensor of a plan's list. Its elements are cut into `chunks`, one to a workgroup.
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
    int32_t filled;    // tensors with any elements
    int32_t chunk;     // elements of one, a multiple of kGradStep
    int32_t norm;      // a lamb_norm
    int64_t bytes;     // of all gradients
    double *partials;  // [chunks]
    double *powers;    // [n]: sums of squares or magnitudes, or the largest magnitude
    uint32_t *done;    // [n + 1], 0 between calls: a tensor's finished chunks; the tensors
};

constexpr int kGradBlock = 256;
constexpr int kGradStep = kGradBlock * 8;  // elements that a chunk is a multiple of
constexpr int kGradTurn = 8 * kGradStep;   // those that a workgroup has in flight

// Lists of up to this many chunks are joined by the launch that sums them: 10 to 11 us for
// the norm of 0.1M to 4M elements, where two launches take 13 (the second costs the host
// 3.5). With more workgroups their arrivals at one counter cost more than that: 14 us for
// 1000 chunks.
constexpr int32_t kGradJoined = 640;

// Gradients that are read again right after (`again`) and of which the last-level cache
// (256 MB) holds a good part are loaded into it, others past it (nontemporal loads): clipping
// 240 MB takes 105 us so and 111 the other way, 400 MB 166 and 176, 560 MB 237 and 239, but
// 1.6 GB 706 and 665; a norm by itself 40.8 us for 200 MB where its loads are kept, 36.8
// where not.
constexpr int64_t kGradKept = int64_t(768) << 20;

hipError_t launch_grad_norms(const GradList &list, bool again, double *norms, double *total,
                             hipStream_t stream);
// out = scale min(1, max_norm / (|scale| total)) in, or scale in where total is not finite.
hipError_t launch_grad_clip(const GradList &list, const double *total, double max_norm,
                            double scale, int32_t *nonfinite_out, hipStream_t stream);

}  // namespace lamb_mi355x
