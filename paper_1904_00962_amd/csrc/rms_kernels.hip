// Root-mean-square norm of rows with the residual's addition before it, its result in 8
// bits with scales, and its gradients, for gfx950.
//
//   h = x + residual, rounded to the residual's type (h = x without one)
//   y = h r w,  r = (mean(h^2) + eps)^-1/2
//   8 bits: s = max(max |y| / 448, 2^-126) over a row or a group of columns, q = e4m3(y / s)
//   backward, with g = dy w: dh = r (g - h r mean(g h r)) + ds,  dw = sum of dy h r
//
// All of it is bound by HBM: a row is read once, stays in the registers of its team's
// lanes, eight columns to a lane, and its results leave from there. The sums of a row are
// taken in fp64, which costs nothing beside the loads and lets no square pass fp32's range.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ops_host.h"
#include "rms_internal.h"
#include "row_io.h"

namespace lamb_mi355x {
namespace {

constexpr float kLargestE4m3 = 448.0f;
constexpr float kLeastScale = 0x1p-126f;

template <class T>
__device__ inline T wave_sum(T v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// The bits of |v| as integers have the order of their values, and NaN above all.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

constexpr int rms_block(int waves) { return 64 * (waves < kRmsWaves ? kRmsWaves : waves); }

// W waves to a row, V times 512 W columns. With QUANT the result is 8 bits wide.
template <int W, int V, bool X_BF16, bool RES, bool RES_BF16, bool QUANT>
__global__ __launch_bounds__(rms_block(W)) void rms_kernel(RmsArgs a, RmsOut o) {
    constexpr int kTeams = rms_block(W) / 64 / W;
    __shared__ double part[kTeams][W];
    __shared__ uint32_t top[kTeams][W];
    const int t = threadIdx.x % (64 * W), team = threadIdx.x / (64 * W), wave = t / 64;
    const int64_t row = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * kTeams + team;
    const bool live = row < a.tokens;
    float h[V][8];
    double sum = 0.0;
    if (live) {
        Eight<X_BF16> x[V];
        Eight<RES_BF16> r[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * 64 * W + t) * 8;
            x[v] = load_eight<X_BF16>(a.x, row * a.x_stride + c, a.dim - c);
            if (RES)
                r[v] = load_eight<RES_BF16>(a.residual, row * a.residual_stride + c, a.dim - c);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * 64 * W + t) * 8;
            x[v].get(h[v]);
            if (RES) {
                float with[8];
                r[v].get(with);
#pragma unroll
                for (int i = 0; i < 8; ++i) with[i] += h[v][i];
                r[v].set(with);
                r[v].get(h[v]);
                if (o.summed)
                    store_eight<RES_BF16, true>(o.summed, row * o.summed_stride + c, a.dim - c, r[v]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma(double(h[v][i]), double(h[v][i]), sum);
        }
        sum = wave_sum(sum);
    }
    if (W > 1) {
        if (t % 64 == 0)
            part[team][wave] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) sum += part[team][w];
    }
    const float inverse = float(1.0 / sqrt(sum / a.dim + double(a.eps)));
    uint32_t largest = 0;
    if (live) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * 64 * W + t) * 8;
            const int n = a.dim - c;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] *= inverse;
            if (a.weight) {
                float w[8];
                load_values(a.weight_bf16, a.weight, c, n, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] *= w[i];
            }
            if (!QUANT) {
                store_values<true>(o.out_bf16, o.out, row * o.out_stride + c, n, h[v]);
            } else if (o.group == 0) {
                // columns past the row are 0 inverse, which may be NaN
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n)
                        largest = max(largest, magnitude(h[v][i]));
            }
        }
    }
    if (!QUANT)
        return;
    if (o.group == 0) {
#pragma unroll
        for (int d = 32; d; d >>= 1) largest = max(largest, uint32_t(__shfl_xor(int(largest), d)));
        if (W > 1) {
            if (t % 64 == 0)
                top[team][wave] = largest;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) largest = max(largest, top[team][w]);
        }
    }
    if (!live)
        return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * 64 * W + t) * 8;
        const int n = a.dim - c;
        if (o.group) {
            largest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n)
                    largest = max(largest, magnitude(h[v][i]));
            for (int d = 1; d < o.group / 8; d <<= 1)
                largest = max(largest, uint32_t(__shfl_xor(int(largest), d)));
        }
        const float most = __uint_as_float(largest) / kLargestE4m3;
        const float scale = most < kLeastScale ? kLeastScale : most;  // NaN stays
        if (n <= 0)
            continue;
        if (o.group ? c % o.group == 0 : c == 0)
            o.scales[row * o.groups + (o.group ? c / o.group : 0)] = scale;
        uint32_t q[2] = {};
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            int word = 0;
            word = __builtin_amdgcn_cvt_pk_fp8_f32(h[v][i] / scale, h[v][i + 1] / scale, word,
                                                   false);
            word = __builtin_amdgcn_cvt_pk_fp8_f32(h[v][i + 2] / scale, h[v][i + 3] / scale, word,
                                                   true);
            q[i / 4] = uint32_t(word);
        }
        uint8_t *p = (uint8_t *)o.out + row * o.out_stride + c;
        if (n >= 8) {
            __builtin_memcpy(p, q, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n)
                    p[i] = uint8_t(q[i / 4] >> (i % 4 * 8));
        }
    }
}

// A team's columns of row after row; what a lane adds to the weight's gradient stays in
// its registers, kRmsFoldRows rows to a sum and these sums to another, and leaves once.
template <int W, bool X_BF16, bool DY_BF16, bool DX_BF16>
__global__ __launch_bounds__(rms_block(W)) void rms_grad_kernel(RmsArgs a, RmsGrad g) {
    constexpr int kTeams = rms_block(W) / 64 / W;
    __shared__ double part[2][kTeams][W][2];
    const int t = threadIdx.x % (64 * W), team = threadIdx.x / (64 * W), wave = t / 64;
    const int c = t * 8, n = a.dim - c;
    const int64_t step = int64_t(gridDim.x) * kTeams;
    float w[8], recent[8] = {}, dw[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.0f;
    if (a.weight)
        load_values(a.weight_bf16, a.weight, c, n, w);
    int rows = 0;
    // every team of a workgroup makes as many turns
    for (int64_t first = int64_t(blockIdx.x) * kTeams; first < a.tokens; first += step) {
        const int64_t row = first + team;
        const bool live = row < a.tokens;
        float x[8] = {}, dy[8] = {}, ds[8] = {}, gw[8];
        if (live) {
            const Eight<X_BF16> xe = load_eight<X_BF16>(a.x, row * a.x_stride + c, n);
            const Eight<DY_BF16> de =
                load_eight<DY_BF16>(g.grad_out, row * g.grad_out_stride + c, n);
            if (g.grad_sum)
                load_eight<DX_BF16>(g.grad_sum, row * g.grad_sum_stride + c, n).get(ds);
            xe.get(x);
            de.get(dy);
        }
        double square = 0.0, along = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gw[i] = dy[i] * w[i];
            square = fma(double(x[i]), double(x[i]), square);
            along = fma(double(x[i]), double(gw[i]), along);
        }
        square = wave_sum(square);
        along = wave_sum(along);
        if (W > 1) {
            double(*to)[2] = part[rows & 1][team];
            if (t % 64 == 0) {
                to[wave][0] = square;
                to[wave][1] = along;
            }
            __syncthreads();
            square = along = 0.0;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                square += to[k][0];
                along += to[k][1];
            }
        }
        const double r = 1.0 / sqrt(square / a.dim + double(a.eps));
        const float inverse = float(r), mean = float(along * r / a.dim);
        if (live) {
            float dx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= inverse;
                dx[i] = fmaf(fmaf(-x[i], mean, gw[i]), inverse, ds[i]);
                recent[i] = fmaf(dy[i], x[i], recent[i]);
            }
            if (g.grad_x) {
                Eight<DX_BF16> e;
                e.set(dx);
                store_eight<DX_BF16, true>(g.grad_x, row * g.grad_x_stride + c, n, e);
            }
        }
        if (++rows % kRmsFoldRows == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] += recent[i];
                recent[i] = 0.0f;
            }
        }
    }
    if (g.grad_weight && n > 0) {
        Eight<false> e;
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] += recent[i];
        e.set(dw);
        store_eight<false>(g.partial, (int64_t(blockIdx.x) * kTeams + team) * g.columns + c, 8, e);
    }
}

// Rows too wide for one lane's registers: first each row's two numbers, a workgroup a row.
__global__ __launch_bounds__(1024) void rms_stats_kernel(RmsArgs a, RmsGrad g) {
    __shared__ double part[16][2];
    const int64_t row = int64_t(blockIdx.y) * gridDim.x + blockIdx.x;
    if (row >= a.tokens)
        return;
    double square = 0.0, along = 0.0;
    for (int c = threadIdx.x * 8; c < a.dim; c += 8192) {
        const int n = a.dim - c;
        float x[8], dy[8], w[8];
        load_values(a.x_bf16, a.x, row * a.x_stride + c, n, x);
        load_values(g.grad_out_bf16, g.grad_out, row * g.grad_out_stride + c, n, dy);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.0f;
        if (a.weight)
            load_values(a.weight_bf16, a.weight, c, n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            square = fma(double(x[i]), double(x[i]), square);
            along = fma(double(x[i]), double(dy[i] * w[i]), along);
        }
    }
    square = wave_sum(square);
    along = wave_sum(along);
    if (threadIdx.x % 64 == 0) {
        part[threadIdx.x / 64][0] = square;
        part[threadIdx.x / 64][1] = along;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        square = along = 0.0;
        for (int k = 0; k < 16; ++k) {
            square += part[k][0];
            along += part[k][1];
        }
        const double r = 1.0 / sqrt(square / a.dim + double(a.eps));
        g.stats[2 * row] = float(r);
        g.stats[2 * row + 1] = float(along * r / a.dim);
    }
}

// Then 2048 columns of kRmsWideRows rows in a workgroup.
__global__ __launch_bounds__(256) void rms_wide_grad_kernel(RmsArgs a, RmsGrad g) {
    const int c = (int(blockIdx.y) * 256 + threadIdx.x) * 8, n = a.dim - c;
    if (n <= 0)
        return;
    float w[8], recent[8] = {}, dw[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.0f;
    if (a.weight)
        load_values(a.weight_bf16, a.weight, c, n, w);
    const int64_t first = int64_t(blockIdx.x) * kRmsWideRows;
    const int64_t end = first + kRmsWideRows < a.tokens ? first + kRmsWideRows : a.tokens;
    for (int64_t row = first; row < end; ++row) {
        float x[8], dy[8], ds[8] = {}, dx[8];
        load_values(a.x_bf16, a.x, row * a.x_stride + c, n, x);
        load_values(g.grad_out_bf16, g.grad_out, row * g.grad_out_stride + c, n, dy);
        if (g.grad_sum)
            load_values(g.grad_x_bf16, g.grad_sum, row * g.grad_sum_stride + c, n, ds);
        const float inverse = g.stats[2 * row], mean = g.stats[2 * row + 1];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= inverse;
            dx[i] = fmaf(fmaf(-x[i], mean, dy[i] * w[i]), inverse, ds[i]);
            recent[i] = fmaf(dy[i], x[i], recent[i]);
        }
        if (g.grad_x)
            store_values(g.grad_x_bf16, g.grad_x, row * g.grad_x_stride + c, n, dx);
        if ((row - first) % kRmsFoldRows == kRmsFoldRows - 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] += recent[i];
                recent[i] = 0.0f;
            }
        }
    }
    if (g.grad_weight) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] += recent[i];
        Eight<false> e;
        e.set(dw);
        store_eight<false>(g.partial, int64_t(blockIdx.x) * g.columns + c, 8, e);
    }
}

// The weight's gradient: its parts in their order, 32 stripes of them and 32 columns in a
// workgroup, in fp64.
__global__ __launch_bounds__(1024) void rms_join_kernel(RmsArgs a, RmsGrad g) {
    __shared__ double part[32][32];
    const int column = threadIdx.x % 32, stripe = threadIdx.x / 32;
    const int c = int(blockIdx.x) * 32 + column;
    double sum = 0.0;
    if (c < a.dim) {
#pragma unroll 8
        for (int64_t k = stripe; k < g.partials; k += 32) sum += double(g.partial[k * g.columns + c]);
    }
    part[stripe][column] = sum;
    __syncthreads();
    if (stripe == 0 && c < a.dim) {
        sum = 0.0;
        for (int k = 0; k < 32; ++k) sum += part[k][column];
        if (g.grad_weight_bf16) {
            __bf16 *to = (__bf16 *)g.grad_weight + c;
            if (g.add_weight)
                sum += double(float(*to));
            *to = __bf16(float(sum));
        } else {
            float *to = (float *)g.grad_weight + c;
            if (g.add_weight)
                sum += double(*to);
            *to = float(sum);
        }
    }
}

int waves_of(int32_t dim) {
    for (int w = 1; w < kRmsMaxWaves; w *= 2)
        if (dim <= 512 * w)
            return w;
    return kRmsMaxWaves;
}

template <bool X_BF16, bool RES, bool RES_BF16, bool QUANT>
hipError_t launch_rms_of(const RmsArgs &a, const RmsOut &o, hipStream_t stream) {
    auto run = [&](auto waves, auto times) {
        constexpr int W = decltype(waves)::value, V = decltype(times)::value;
        constexpr int kTeams = rms_block(W) / 64 / W;
        rms_kernel<W, V, X_BF16, RES, RES_BF16, QUANT>
            <<<grid_of((a.tokens + kTeams - 1) / kTeams), rms_block(W), 0, stream>>>(a, o);
        return hipGetLastError();
    };
    std::integral_constant<int, 1> c1;
    std::integral_constant<int, 2> c2;
    std::integral_constant<int, 4> c4;
    std::integral_constant<int, 8> c8;
    std::integral_constant<int, 16> c16;
    switch (waves_of(a.dim)) {
    case 1: return run(c1, c1);
    case 2: return run(c2, c1);
    case 4: return run(c4, c1);
    case 8: return run(c8, c1);
    }
    if (a.dim <= 8192)
        return run(c16, c1);
    if (a.dim <= 16384)
        return run(c16, c2);
    return a.dim <= 32768 ? run(c16, c4) : run(c16, c8);
}

template <bool QUANT>
hipError_t launch_rms_types(const RmsArgs &a, const RmsOut &o, hipStream_t stream) {
    if (!a.residual)
        return a.x_bf16 ? launch_rms_of<true, false, true, QUANT>(a, o, stream)
                        : launch_rms_of<false, false, false, QUANT>(a, o, stream);
    if (!a.x_bf16)
        return launch_rms_of<false, true, false, QUANT>(a, o, stream);
    return a.residual_bf16 ? launch_rms_of<true, true, true, QUANT>(a, o, stream)
                           : launch_rms_of<true, true, false, QUANT>(a, o, stream);
}

int64_t grad_blocks(int64_t tokens, int32_t dim) {
    const int waves = waves_of(dim);
    const int64_t teams = rms_block(waves) / 64 / waves;
    const int64_t all = (tokens + teams - 1) / teams;
    return std::min<int64_t>(all, 4096 / (rms_block(waves) / 64));
}

template <bool X_BF16, bool DY_BF16, bool DX_BF16>
hipError_t launch_rms_grad_of(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    auto run = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        rms_grad_kernel<W, X_BF16, DY_BF16, DX_BF16>
            <<<uint32_t(grad_blocks(a.tokens, a.dim)), rms_block(W), 0, stream>>>(a, g);
        return hipGetLastError();
    };
    switch (waves_of(a.dim)) {
    case 1: return run(std::integral_constant<int, 1>{});
    case 2: return run(std::integral_constant<int, 2>{});
    case 4: return run(std::integral_constant<int, 4>{});
    case 8: return run(std::integral_constant<int, 8>{});
    default: return run(std::integral_constant<int, 16>{});
    }
}

}  // namespace

hipError_t launch_rms(const RmsArgs &args, const RmsOut &out, hipStream_t stream) {
    return out.scales ? launch_rms_types<true>(args, out, stream)
                      : launch_rms_types<false>(args, out, stream);
}

int64_t rms_partials(int64_t tokens, int32_t dim) {
    if (dim > kRmsHeldDim)
        return (tokens + kRmsWideRows - 1) / kRmsWideRows;
    const int waves = waves_of(dim);
    return grad_blocks(tokens, dim) * (rms_block(waves) / 64 / waves);
}

hipError_t launch_rms_grad(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    if (a.dim > kRmsHeldDim) {
        rms_stats_kernel<<<grid_of(a.tokens), 1024, 0, stream>>>(a, g);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess)
            return err;
        const dim3 grid(uint32_t(g.partials), uint32_t((a.dim + 2047) / 2048));
        rms_wide_grad_kernel<<<grid, 256, 0, stream>>>(a, g);
        return hipGetLastError();
    }
    auto by_dx = [&](auto x, auto dy) {
        constexpr bool X = decltype(x)::value, DY = decltype(dy)::value;
        return g.grad_x_bf16 ? launch_rms_grad_of<X, DY, true>(a, g, stream)
                             : launch_rms_grad_of<X, DY, false>(a, g, stream);
    };
    auto by_dy = [&](auto x) {
        return g.grad_out_bf16 ? by_dx(x, std::true_type{}) : by_dx(x, std::false_type{});
    };
    return a.x_bf16 ? by_dy(std::true_type{}) : by_dy(std::false_type{});
}

hipError_t launch_rms_join(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    rms_join_kernel<<<uint32_t((a.dim + 31) / 32), 1024, 0, stream>>>(a, g);
    return hipGetLastError();
}

}  // namespace lamb_mi355x
