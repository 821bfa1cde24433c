// Host side of the gradients' norms and clipping, the lamb_grad_* entry points of
// include/lamb_ops.h.
#include <math.h>

#include <algorithm>

#include "gradnorm_internal.h"
#include "ops_host.h"

using namespace lamb_mi355x;

struct lamb_grad_plan {
    int device = 0;
    bool clips = false;
    void *block = nullptr;  // every device buffer of the plan
    GradList list{};
    CallOrder order;
};

namespace {

// Chunks are as long as a workgroup loads at once, half of that where there would be too few
// for all CUs. (4 steps in place of 1: 11 us for the norm of 2M to 4M elements in place of
// 13 to 14, whose time is the joins'. 8 steps in place of 16 or 32, which are further from
// filling a last round: 979 us for 1.56 billion fp32 elements in place of 994 and 1007.)
int32_t pick_chunk(int64_t numel) {
    constexpr int64_t kWorkgroups = 2048, kLeast = 4 * kGradStep, kMost = 8 * kGradStep;
    const int64_t each = round_up((numel + kWorkgroups - 1) / kWorkgroups, kGradStep);
    return int32_t(std::min(std::max(each, kLeast), kMost));
}

lamb_status build(lamb_grad_plan *plan, std::vector<GradTensor> &tensors) {
    GradList &l = plan->list;
    int64_t numel = 0, chunks = 0;
    for (const GradTensor &t : tensors) {
        numel += t.numel;
        l.bytes += t.numel * (t.in_bf16 ? 2 : 4);
    }
    l.chunk = pick_chunk(numel);
    for (GradTensor &t : tensors) {
        const int64_t own = (t.numel + l.chunk - 1) / l.chunk;
        if (chunks + own > INT32_MAX)
            return fail(LAMB_EINVAL, "the tensors take too many chunks for one plan");
        t.first_chunk = int32_t(chunks);
        t.chunks = int32_t(own);
        l.filled += own > 0;
        chunks += own;
    }
    l.n = int32_t(tensors.size());
    l.chunks = int32_t(chunks);
    size_t bytes = 0;
    auto take = [&](size_t size) {
        const size_t at = bytes;
        bytes += size_t(round_up(int64_t(size), 256));
        return at;
    };
    // what the host writes comes first, so that one copy brings it
    const size_t o_tensors = take(tensors.size() * sizeof(GradTensor));
    const size_t o_chunks = take(size_t(chunks) * 4);
    const size_t o_powers = take(tensors.size() * 8);
    const size_t o_done = take((tensors.size() + 1) * 4);
    const size_t written = bytes;
    const size_t o_partials = take(size_t(chunks) * 8);
    std::vector<char> host(written, 0);
    std::copy_n(tensors.data(), tensors.size(),
                reinterpret_cast<GradTensor *>(host.data() + o_tensors));
    int32_t *chunk_tensor = reinterpret_cast<int32_t *>(host.data() + o_chunks);
    for (int32_t i = 0; i < l.n; ++i)
        std::fill_n(chunk_tensor + tensors[i].first_chunk, tensors[i].chunks, i);
    hipError_t err = hipGetDevice(&plan->device);
    if (err != hipSuccess)
        return fail_hip(err, "hipGetDevice");
    // only orders kernels of this device: no system-scope fence
    err = hipEventCreateWithFlags(&plan->order.done,
                                  hipEventDisableTiming | hipEventDisableSystemFence);
    if (err != hipSuccess)
        return fail_hip(err, "hipEventCreateWithFlags");
    err = hipMalloc(&plan->block, bytes);
    if (err != hipSuccess) {
        plan->block = nullptr;
        (void)hipGetLastError();
        return fail(LAMB_ENOMEM, "hipMalloc of %zu bytes: %s", bytes, hipGetErrorString(err));
    }
    char *base = static_cast<char *>(plan->block);
    err = hipMemcpy(base, host.data(), written, hipMemcpyHostToDevice);
    if (err != hipSuccess)
        return fail_hip(err, "hipMemcpy");
    l.tensors = reinterpret_cast<const GradTensor *>(base + o_tensors);
    l.chunk_tensor = reinterpret_cast<const int32_t *>(base + o_chunks);
    l.partials = reinterpret_cast<double *>(base + o_partials);
    l.powers = reinterpret_cast<double *>(base + o_powers);
    l.done = reinterpret_cast<uint32_t *>(base + o_done);
    return LAMB_OK;
}

lamb_status check_totals(const lamb_grad_plan *plan, const double *norms, const double *total) {
    if (!plan || !total)
        return fail(LAMB_ENULL, "plan and total must not be NULL");
    if (!aligned_to(norms, 8) || !aligned_to(total, 8))
        return fail(LAMB_EALIGN, "norms and total must be 8-byte aligned");
    return LAMB_OK;
}

lamb_status check_clip(const lamb_grad_plan *plan, const double *total, double max_norm,
                       double scale, const int32_t *nonfinite_out) {
    const lamb_status st = check_totals(plan, nullptr, total);
    if (st != LAMB_OK)
        return st;
    if (!plan->clips)
        return fail(LAMB_EPLAN, "the plan has tensors without an out");
    if (!aligned_to(nonfinite_out, 4))
        return fail(LAMB_EALIGN, "nonfinite_out is not aligned to its element");
    if (!(max_norm >= 0.0))
        return fail(LAMB_EINVAL, "max_norm = %g, need >= 0", max_norm);
    if (!std::isfinite(scale))
        return fail(LAMB_EINVAL, "scale = %g must be finite", scale);
    return LAMB_OK;
}

}  // namespace

extern "C" {

lamb_status lamb_grad_plan_create(const lamb_grad_tensor *tensors, int32_t n, int32_t norm,
                                  lamb_grad_plan **out) {
    if (!out)
        return fail(LAMB_ENULL, "out must not be NULL");
    *out = nullptr;
    if (!tensors)
        return fail(LAMB_ENULL, "tensors must not be NULL");
    if (n < 1)
        return fail(LAMB_EINVAL, "n = %d, need >= 1", n);
    if (norm != LAMB_NORM_L2 && norm != LAMB_NORM_L1 && norm != LAMB_NORM_LINF)
        return fail(LAMB_EINVAL, "unknown norm %d", norm);
    return guarded([&]() -> lamb_status {
        std::vector<GradTensor> list;
        std::vector<Span> spans;
        bool clips = true;
        for (int32_t i = 0; i < n; ++i) {
            const lamb_grad_tensor &t = tensors[i];
            if (t.numel < 0 || t.numel > kMaxNumel)
                return fail(LAMB_EINVAL, "tensor %d has %lld elements, need 0 to 2^40", i,
                            (long long)t.numel);
            if (!is_float(t.in_dtype) || (t.out && !is_float(t.out_dtype)))
                return fail(LAMB_EINVAL, "tensor %d: gradients are float32 or bfloat16", i);
            if (t.numel && !t.in)
                return fail(LAMB_ENULL, "tensor %d: in must not be NULL", i);
            if (!aligned_to(t.in, uintptr_t(size_of(t.in_dtype))) ||
                !aligned_to(t.out, uintptr_t(size_of(t.out_dtype))))
                return fail(LAMB_EALIGN, "tensor %d: a pointer is not aligned to its elements", i);
            clips &= t.out || t.numel == 0;
            const uint64_t in_bytes = uint64_t(t.numel * size_of(t.in_dtype));
            if (t.in != t.out || t.in_dtype != t.out_dtype)
                spans.push_back(span_of(t.in, in_bytes, false, i, "in"));
            if (t.out)
                spans.push_back(span_of(t.out, uint64_t(t.numel * size_of(t.out_dtype)), true, i,
                                        "out"));
            list.push_back(GradTensor{t.in, t.out, t.numel, t.in_dtype == LAMB_DTYPE_BF16,
                                      t.out_dtype == LAMB_DTYPE_BF16, 0, 0});
        }
        lamb_status s = check_spans(spans.data(), spans.size());
        if (s != LAMB_OK)
            return s;
        lamb_grad_plan *plan = new lamb_grad_plan;
        plan->clips = clips;
        plan->list.norm = norm;
        s = guarded([&] { return build(plan, list); });
        if (s != LAMB_OK) {
            (void)lamb_grad_plan_destroy(plan);
            return s;
        }
        *out = plan;
        return LAMB_OK;
    });
}

lamb_status lamb_grad_norm(lamb_grad_plan *plan, double *norms, double *total, void *stream_in) {
    const lamb_status st = check_totals(plan, norms, total);
    if (st != LAMB_OK)
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    DeviceScope scope(plan->device);
    return ordered(plan->order, stream, [&] {
        const hipError_t err = launch_grad_norms(plan->list, false, norms, total, stream);
        return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
    });
}

lamb_status lamb_grad_clip(lamb_grad_plan *plan, const double *total, double max_norm,
                           double scale, int32_t *nonfinite_out, void *stream_in) {
    const lamb_status st = check_clip(plan, total, max_norm, scale, nonfinite_out);
    if (st != LAMB_OK)
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    DeviceScope scope(plan->device);
    return ordered(plan->order, stream, [&] {
        const hipError_t err =
            launch_grad_clip(plan->list, total, max_norm, scale, nonfinite_out, stream);
        return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
    });
}

lamb_status lamb_grad_norm_clip(lamb_grad_plan *plan, double *norms, double *total,
                                double max_norm, double scale, int32_t *nonfinite_out,
                                void *stream_in) {
    lamb_status st = check_totals(plan, norms, total);
    if (st == LAMB_OK)
        st = check_clip(plan, total, max_norm, scale, nonfinite_out);
    if (st != LAMB_OK)
        return st;
    hipStream_t stream = static_cast<hipStream_t>(stream_in);
    DeviceScope scope(plan->device);
    return ordered(plan->order, stream, [&] {
        hipError_t err = launch_grad_norms(plan->list, true, norms, total, stream);
        if (err == hipSuccess)
            err = launch_grad_clip(plan->list, total, max_norm, scale, nonfinite_out, stream);
        return err == hipSuccess ? LAMB_OK : fail_hip(err, "kernel launch");
    });
}

lamb_status lamb_grad_plan_destroy(lamb_grad_plan *plan) {
    if (!plan)
        return LAMB_OK;
    DeviceScope scope(plan->device);
    hipError_t err = plan->block ? hipFree(plan->block) : hipSuccess;  // waits for its users
    const hipError_t event = plan->order.done ? hipEventDestroy(plan->order.done) : hipSuccess;
    if (err == hipSuccess)
        err = event;
    delete plan;
    if (err != hipSuccess)
        return fail_hip(err, "hipFree, hipEventDestroy");
    return LAMB_OK;
}

}  // extern "C"
