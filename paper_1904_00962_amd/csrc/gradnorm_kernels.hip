// Norms of a list of gradient tensors, and the list scaled to keep a limit, for gfx950.
//
// Bound by HBM: each pass reads every gradient once. Sums are taken in fp64, element by
// element, so that neither squares nor long sums lose anything, and in a fixed order: a
// chunk's, a tensor's chunks, the tensors.
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

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

    template <int N>
    __device__ inline void elements(const float (&g)[N]) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (NORM == LAMB_NORM_L2)
                v = fma(double(g[i]), double(g[i]), v);
            else if (NORM == LAMB_NORM_L1)
                v += fabs(double(g[i]));
            else
                top = max(top, __float_as_uint(g[i]) & 0x7fffffffu);
        }
        if (NORM == LAMB_NORM_LINF)
            join(double(__uint_as_float(top)));
    }
    __device__ inline void join(double w) {
        if (NORM != LAMB_NORM_LINF)
            v += w;
        else if (__double_as_longlong(w) > __double_as_longlong(v))
            v = w;
    }
    __device__ inline double norm() const { return NORM == LAMB_NORM_L2 ? sqrt(v) : v; }
};

// The workgroup's, on thread 0.
template <int NORM>
__device__ inline void join_block(Power<NORM> &power, double *shared) {
#pragma unroll
    for (int d = 32; d; d >>= 1) power.join(__shfl_xor(power.v, d));
    __syncthreads();  // who read `shared` before has done so
    if (threadIdx.x % 64 == 0)
        shared[threadIdx.x / 64] = power.v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kGradBlock / 64; ++w) power.join(shared[w]);
}

// A lane's 16 bytes of a gradient tensor, which follow one another over the lanes.
template <bool BF16>
struct Part {
    static constexpr int kElements = BF16 ? 8 : 4;
    Bytes16 u;

    __device__ inline void get(float (&v)[kElements]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                v[2 * i] = bf16_low(u[i]);
                v[2 * i + 1] = bf16_high(u[i]);
            } else {
                v[i] = __uint_as_float(u[i]);
            }
        }
    }
};

template <bool BF16, bool STREAM>
__device__ inline Part<BF16> load_part(const void *base, int64_t at) {
    using T = typename std::conditional<BF16, uint16_t, uint32_t>::type;
    return Part<BF16>{load_16<STREAM>((const Global<T> *)base + at)};
}

// The first n elements of one; 0 past them.
template <bool BF16>
__device__ inline Part<BF16> load_some(const void *base, int64_t at, int n) {
    using T = typename std::conditional<BF16, uint16_t, uint32_t>::type;
    const Global<T> *p = (const Global<T> *)base + at;
    Part<BF16> e = {};
#pragma unroll
    for (int i = 0; i < Part<BF16>::kElements; ++i)
        if (i < n)
            e.u[BF16 ? i / 2 : i] |= uint32_t(p[i]) << (BF16 ? i % 2 * 16 : 0);
    return e;
}

// Adds the elements from `first` to `end`: a whole chunk's, or half of one's, in flight at
// once (short lists have chunks of half the length and more).
template <int NORM, bool BF16, bool STREAM>
__device__ inline void add_elements(Power<NORM> &power, const void *in, int64_t first,
                                    int64_t end) {
    constexpr int kEach = Part<BF16>::kElements, kAcross = kGradBlock * kEach;
    float v[kEach];
    int64_t at = first + threadIdx.x * kEach;
    auto turns = [&](auto size) {
        constexpr int kTurn = decltype(size)::value, kParts = kTurn / kAcross;
        for (; first + kTurn <= end; first += kTurn, at += kTurn) {
            Part<BF16> e[kParts];
#pragma unroll
            for (int k = 0; k < kParts; ++k) e[k] = load_part<BF16, STREAM>(in, at + k * kAcross);
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                e[k].get(v);
                power.elements(v);
            }
        }
    };
    turns(std::integral_constant<int, kGradTurn>{});
    turns(std::integral_constant<int, kGradTurn / 2>{});
    turns(std::integral_constant<int, kGradTurn / 8>{});
    for (; at < end; at += kAcross) {
        const int64_t n = end - at;
        (n < kEach ? load_some<BF16>(in, at, int(n)) : load_part<BF16, false>(in, at)).get(v);
        power.elements(v);
    }
}

// The elements of a chunk, from `first` to `end` of its tensor.
struct Chunk {
    GradTensor t;
    int32_t tensor;
    int64_t first, end;

    __device__ inline Chunk(const GradList &l, int64_t chunk) {
        tensor = l.chunk_tensor[chunk];
        t = l.tensors[tensor];
        first = (chunk - t.first_chunk) * l.chunk;
        end = first + l.chunk < t.numel ? first + l.chunk : t.numel;
    }
};

template <int NORM, bool STREAM>
__device__ inline void add_chunk(Power<NORM> &power, const Chunk &c) {
    if (c.t.in_bf16)
        add_elements<NORM, true, STREAM>(power, c.t.in, c.first, c.end);
    else
        add_elements<NORM, false, STREAM>(power, c.t.in, c.first, c.end);
}

// Whether this workgroup, of `all`, is the last to come here; the counter is then 0 again
// (it wraps by itself, so it is also after calls that wrongly ran beside each other). What
// thread 0 of the others has put() before it came, this one can take(): those are accesses
// at device scope, past the caches that the dies do not share, and thread 0 waits for its
// own to end. A release fence in its place writes a die's whole L2 back, for each
// workgroup: 400 us in place of 125 for the norms of 335M bf16 elements.
__device__ inline bool last_of(uint32_t *counter, uint32_t all, uint32_t *shared) {
    __syncthreads();  // who read `shared` before has done so
    if (threadIdx.x == 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        *shared = atomicInc(counter, all - 1) == all - 1;
    }
    __syncthreads();
    return *shared;
}

__device__ inline void put(double *to, double v) {
    __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline double take(const double *from) {
    return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int NORM>
__device__ inline void put_power(const GradList &l, int32_t i, const Power<NORM> &power,
                                 double *norms) {
    if (threadIdx.x != 0)
        return;
    put(&l.powers[i], power.v);
    if (norms)
        norms[i] = power.norm();
}

template <int NORM>
__device__ inline void join_tensors(const GradList &l, double *norms, double *total,
                                    double *shared) {
    Power<NORM> power;
    for (int k = threadIdx.x; k < l.n; k += kGradBlock) {
        power.join(take(&l.powers[k]));
        if (norms && l.filled < l.n && l.tensors[k].numel == 0)
            norms[k] = 0.0;
    }
    join_block(power, shared);
    if (threadIdx.x == 0)
        *total = power.norm();
}

template <int NORM>
__device__ inline void join_chunks(const GradList &l, int32_t first, int32_t chunks,
                                   Power<NORM> &power, double *shared) {
    power = Power<NORM>();
#pragma unroll 4
    for (int k = threadIdx.x; k < chunks; k += kGradBlock)
        power.join(take(&l.partials[first + k]));
    join_block(power, shared);
}

// A chunk's sum. In short lists (JOIN) the last workgroup at a tensor joins the tensor's
// chunks, the last of all the tensors: no second launch, and no workgroup waits for another.
// STREAM: loads past the caches.
//
// Bound by HBM: 6.23 GB of fp32 in 930 us, 6.7 TB/s (980 with eight elements a lane); 670 MB
// of bf16 in 96 to 98 us, 6.9 (some of it from the last-level cache). Chunks follow one
// another over the workgroups: with one long range to a workgroup, so that fewer sums were
// joined, the dies' 2048 streams took 1.10 ms and 104 us. 2.4 MB in 8 tensors take 6.3 us,
// joins included: latency.
template <int NORM, bool JOIN, bool STREAM>
__global__ __launch_bounds__(kGradBlock) void grad_norms_kernel(GradList l, double *norms,
                                                                double *total) {
    __shared__ double part[kGradBlock / 64];
    __shared__ uint32_t last;
    const int64_t chunk = int64_t(blockIdx.y) * gridDim.x + blockIdx.x;
    if (chunk >= l.chunks)
        return;
    const Chunk c(l, chunk);
    Power<NORM> power;
    add_chunk<NORM, STREAM>(power, c);
    join_block(power, part);
    if (!JOIN) {
        if (threadIdx.x == 0)
            l.partials[chunk] = power.v;
        return;
    }
    if (c.t.chunks > 1) {
        if (threadIdx.x == 0)
            put(&l.partials[chunk], power.v);
        if (!last_of(&l.done[c.tensor], uint32_t(c.t.chunks), &last))
            return;
        join_chunks(l, c.t.first_chunk, c.t.chunks, power, part);
    }
    put_power(l, c.tensor, power, norms);
    if (last_of(&l.done[l.n], uint32_t(l.filled), &last))
        join_tensors<NORM>(l, norms, total, part);
}

// The joins of long lists: a workgroup's tensors one after another. 8 us for 391 tensors, 11
// for 580: latency. (One workgroup for all took 28 and 61.)
template <int NORM>
__global__ __launch_bounds__(kGradBlock) void grad_totals_kernel(GradList l, double *norms,
                                                                 double *total) {
    __shared__ double part[kGradBlock / 64];
    __shared__ uint32_t last;
    for (int32_t i = blockIdx.x; i < l.n; i += gridDim.x) {
        const int32_t first = l.tensors[i].first_chunk, chunks = l.tensors[i].chunks;
        Power<NORM> power;
        join_chunks(l, first, chunks, power, part);
        put_power(l, i, power, norms);
    }
    if (last_of(&l.done[l.n], gridDim.x, &last))
        join_tensors<NORM>(l, norms, total, part);
}

// Of lists without any element.
__global__ __launch_bounds__(kGradBlock) void grad_zeros_kernel(int32_t n, double *norms,
                                                                double *total) {
    if (threadIdx.x == 0)
        *total = 0.0;
    if (norms)
        for (int i = threadIdx.x; i < n; i += kGradBlock) norms[i] = 0.0;
}

// Eight elements a lane, whatever the types: with 16 bytes of fp32 a lane, as the norms have
// it, their four bf16 results took 1750 us in place of 1630 for the case below.
// F: float, or double for factors that fp32 does not hold.
template <bool IN_BF16, bool OUT_BF16, class F>
__device__ inline void scale_chunk(const Chunk &c, F f) {
    auto scaled = [&](const Eight<IN_BF16> &e) {
        float v[8];
        e.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = float(F(v[i]) * f);
        Eight<OUT_BF16> to;
        to.set(v);
        return to;
    };
    int64_t first = c.first, at = first + threadIdx.x * 8;
    auto turns = [&](auto size) {
        constexpr int kTurn = decltype(size)::value, kParts = kTurn / kGradStep;
        for (; first + kTurn <= c.end; first += kTurn, at += kTurn) {
            Eight<IN_BF16> e[kParts];
#pragma unroll
            for (int k = 0; k < kParts; ++k)
                e[k] = load_eight<IN_BF16, false>(c.t.in, at + k * kGradStep, 8);
#pragma unroll
            for (int k = 0; k < kParts; ++k)
                store_eight<OUT_BF16, false, true>(c.t.out, at + k * kGradStep, 8, scaled(e[k]));
        }
    };
    if constexpr (std::is_same<F, float>::value) {
        turns(std::integral_constant<int, kGradTurn>{});
        turns(std::integral_constant<int, kGradTurn / 2>{});
    }
    for (; at < c.end; at += kGradStep) {
        const int n = int(c.end - at < 8 ? c.end - at : 8);
        store_eight<OUT_BF16, true>(c.t.out, at, n,
                                    scaled(load_eight<IN_BF16, true>(c.t.in, at, n)));
    }
}

template <class F>
__device__ inline void scale_chunk(const Chunk &c, F f) {
    if (c.t.in_bf16) {
        if (c.t.out_bf16)
            scale_chunk<true, true>(c, f);
        else
            scale_chunk<true, false>(c, f);
    } else {
        if (c.t.out_bf16)
            scale_chunk<false, true>(c, f);
        else
            scale_chunk<false, false>(c, f);
    }
}

// The last chunks first: the norms have left them in the last-level cache. Bound by HBM: 1.56
// billion fp32 to bf16, 9.35 GB in 1.63 ms, 5.7 TB/s. Eight loads ahead in place of four: 1740
// to 1630 us; results past the caches: 3% less for all sizes.
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
    const double f = finite && fabs(scale) * norm > max_norm ? copysign(max_norm / norm, scale)
                                                             : scale;
    const float rounded = float(f);
    const Chunk c(l, l.chunks - 1 - block);
    if (rounded == 1.0f && c.t.in == c.t.out)
        return;
    // Outside its normal range fp32 would round f by more than its half step, to 0 or to
    // infinity: gradients of 1e38 have norms of 1e43.
    if (f == 0.0 || (fabs(f) >= 0x1p-126 && isfinite(rounded)))
        scale_chunk(c, rounded);
    else
        scale_chunk(c, f);
}

template <int NORM>
hipError_t launch_norms_of(const GradList &l, bool again, double *norms, double *total,
                           hipStream_t stream) {
    if (l.chunks <= kGradJoined) {
        grad_norms_kernel<NORM, true, false>
            <<<uint32_t(l.chunks), kGradBlock, 0, stream>>>(l, norms, total);
        return hipGetLastError();
    }
    auto kernel = again && l.bytes <= kGradKept ? grad_norms_kernel<NORM, false, false>
                        : grad_norms_kernel<NORM, false, true>;
    kernel<<<grid_of(l.chunks), kGradBlock, 0, stream>>>(l, norms, total);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    const uint32_t blocks = uint32_t(l.n < 1024 ? l.n : 1024);
    grad_totals_kernel<NORM><<<blocks, kGradBlock, 0, stream>>>(l, norms, total);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_norms(const GradList &l, bool again, double *norms, double *total,
                             hipStream_t stream) {
    if (l.chunks == 0) {
        grad_zeros_kernel<<<1, kGradBlock, 0, stream>>>(l.n, norms, total);
        return hipGetLastError();
    }
    switch (l.norm) {
    case LAMB_NORM_L2: return launch_norms_of<LAMB_NORM_L2>(l, again, norms, total, stream);
    case LAMB_NORM_L1: return launch_norms_of<LAMB_NORM_L1>(l, again, norms, total, stream);
    default: return launch_norms_of<LAMB_NORM_LINF>(l, again, norms, total, stream);
    }
}

hipError_t launch_grad_clip(const GradList &l, const double *total, double max_norm, double scale,
                            int32_t *nonfinite_out, hipStream_t stream) {
    grad_clip_kernel<<<grid_of(l.chunks ? l.chunks : 1), kGradBlock, 0, stream>>>(
        l, total, max_norm, scale, nonfinite_out);
    return hipGetLastError();
}

}  // namespace lamb_mi355x
