// Norms of a list of gradient tensors, and the list scaled to keep a limit, for gfx950.
//
// Bound by HBM: each pass reads every gradient once. Sums are taken in fp64, element by
// element, so that neither squares nor long sums lose anything, and in a fixed order: a
// workgroup's chunk, a tensor's chunks, the tensors.
#include <hip/hip_runtime.h>
#include <math.h>

#include "gradnorm_internal.h"
#include "ops_host.h"
#include "row_io.h"

namespace lamb_mi355x {
namespace {

// Of L2, L1 and the largest magnitude: what an element adds, and how parts join. The bits
// of a magnitude as integers have the order of the values, with NaN above all, so NaN is
// the largest.
template <int NORM>
struct Power {
    double v = 0.0;

    __device__ inline void element(float g) {
        if (NORM == LAMB_NORM_L2)
            v = fma(double(g), double(g), v);
        else
            join(fabs(double(g)));
    }
    __device__ inline void join(double w) {
        if (NORM != LAMB_NORM_LINF)
            v += w;
        else if (__double_as_longlong(w) > __double_as_longlong(v))
            v = w;
    }
    __device__ inline double norm() const { return NORM == LAMB_NORM_L2 ? sqrt(v) : v; }
    __device__ inline void join_wave() {
#pragma unroll
        for (int d = 32; d; d >>= 1) join(__shfl_xor(v, d));
    }
};

template <int NORM, bool BF16>
__device__ inline Power<NORM> chunk_power(const GradTensor &t, int64_t first, int64_t end) {
    constexpr int kAhead = 4;
    Power<NORM> power;
    int64_t at = first + threadIdx.x * 8;
    for (; at + (kAhead - 1) * kGradStep + 8 <= end; at += kAhead * kGradStep) {
        Eight<BF16> e[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) e[k] = load_eight<BF16>(t.in, at + k * kGradStep, 8);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float v[8];
            e[k].get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) power.element(v[i]);
        }
    }
    for (; at < end; at += kGradStep) {
        float v[8];
        load_eight<BF16>(t.in, at, int(end - at < 8 ? end - at : 8)).get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) power.element(v[i]);  // 0 past the end
    }
    return power;
}

// A chunk's tensor, and its elements from `first` to `end`.
__device__ inline GradTensor chunk_of(const GradList &l, int64_t chunk, int64_t *first,
                                      int64_t *end) {
    GradTensor t = l.tensors[l.chunk_tensor[chunk]];
    t.in = in_device_memory(t.in);
    t.out = in_device_memory(t.out);
    *first = (chunk - t.first_chunk) * l.chunk;
    *end = *first + l.chunk < t.numel ? *first + l.chunk : t.numel;
    return t;
}

template <int NORM>
__global__ __launch_bounds__(kGradBlock) void grad_norms_kernel(GradList l) {
    __shared__ double part[kGradBlock / 64];
    const int64_t chunk = int64_t(blockIdx.y) * gridDim.x + blockIdx.x;
    if (chunk >= l.chunks)
        return;
    int64_t first, end;
    const GradTensor t = chunk_of(l, chunk, &first, &end);
    Power<NORM> power = t.in_bf16 ? chunk_power<NORM, true>(t, first, end)
                                  : chunk_power<NORM, false>(t, first, end);
    power.join_wave();
    if (threadIdx.x % 64 == 0)
        part[threadIdx.x / 64] = power.v;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kGradBlock / 64; ++w) power.join(part[w]);
        l.partials[chunk] = power.v;
    }
}

// One workgroup: each tensor's chunks by a wave, then all tensors.
template <int NORM>
__global__ __launch_bounds__(1024) void grad_totals_kernel(GradList l, double *norms,
                                                           double *total) {
    __shared__ double part[16];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int i = wave; i < l.n; i += 16) {
        const int32_t first = l.tensors[i].first_chunk, chunks = l.tensors[i].chunks;
        Power<NORM> power;
        for (int k = lane; k < chunks; k += 64) power.join(l.partials[first + k]);
        power.join_wave();
        if (lane == 0) {
            l.powers[i] = power.v;
            if (norms)
                norms[i] = power.norm();
        }
    }
    __syncthreads();
    Power<NORM> power;
    for (int i = threadIdx.x; i < l.n; i += 1024) power.join(l.powers[i]);
    power.join_wave();
    if (lane == 0)
        part[wave] = power.v;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) power.join(part[w]);
        *total = power.norm();
    }
}

template <bool IN_BF16, bool OUT_BF16>
__device__ inline void scale_chunk(const GradTensor &t, int64_t first, int64_t end, float f) {
    constexpr int kAhead = 4;
    auto scaled = [&](const Eight<IN_BF16> &e) {
        float v[8];
        e.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= f;
        Eight<OUT_BF16> to;
        to.set(v);
        return to;
    };
    int64_t at = first + threadIdx.x * 8;
    for (; at + (kAhead - 1) * kGradStep + 8 <= end; at += kAhead * kGradStep) {
        Eight<IN_BF16> e[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) e[k] = load_eight<IN_BF16>(t.in, at + k * kGradStep, 8);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            store_eight<OUT_BF16>(t.out, at + k * kGradStep, 8, scaled(e[k]));
    }
    for (; at < end; at += kGradStep) {
        const int n = int(end - at < 8 ? end - at : 8);
        store_eight<OUT_BF16>(t.out, at, n, scaled(load_eight<IN_BF16>(t.in, at, n)));
    }
}

// The last chunks first: the pass before has left them in the last-level cache.
__global__ __launch_bounds__(kGradBlock) void grad_clip_kernel(GradList l, const double *total,
                                                               double max_norm, double scale,
                                                               int32_t *nonfinite_out) {
    const int64_t block = int64_t(blockIdx.y) * gridDim.x + blockIdx.x;
    const double norm = *total;
    const bool finite = isfinite(norm);
    if (block == 0 && threadIdx.x == 0 && nonfinite_out)
        *nonfinite_out = !finite;
    if (block >= l.chunks)
        return;
    const double scaled = fabs(scale) * norm;
    const float f = float(finite && scaled > max_norm ? scale * (max_norm / scaled) : scale);
    int64_t first, end;
    const GradTensor t = chunk_of(l, l.chunks - 1 - block, &first, &end);
    if (f == 1.0f && t.in == t.out)
        return;
    if (t.in_bf16) {
        if (t.out_bf16)
            scale_chunk<true, true>(t, first, end, f);
        else
            scale_chunk<true, false>(t, first, end, f);
    } else {
        if (t.out_bf16)
            scale_chunk<false, true>(t, first, end, f);
        else
            scale_chunk<false, false>(t, first, end, f);
    }
}

}  // namespace

hipError_t launch_grad_norms(const GradList &l, hipStream_t stream) {
    auto kernel = l.norm == LAMB_NORM_L2   ? grad_norms_kernel<LAMB_NORM_L2>
                  : l.norm == LAMB_NORM_L1 ? grad_norms_kernel<LAMB_NORM_L1>
                                           : grad_norms_kernel<LAMB_NORM_LINF>;
    kernel<<<grid_of(l.chunks), kGradBlock, 0, stream>>>(l);
    return hipGetLastError();
}

hipError_t launch_grad_totals(const GradList &l, double *norms, double *total,
                              hipStream_t stream) {
    auto kernel = l.norm == LAMB_NORM_L2   ? grad_totals_kernel<LAMB_NORM_L2>
                  : l.norm == LAMB_NORM_L1 ? grad_totals_kernel<LAMB_NORM_L1>
                                           : grad_totals_kernel<LAMB_NORM_LINF>;
    kernel<<<1, 1024, 0, stream>>>(l, norms, total);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const GradList &l, const double *total, double max_norm, double scale,
                            int32_t *nonfinite_out, hipStream_t stream) {
    grad_clip_kernel<<<grid_of(l.chunks ? l.chunks : 1), kGradBlock, 0, stream>>>(
        l, total, max_norm, scale, nonfinite_out);
    return hipGetLastError();
}

}  // namespace lamb_mi355x
