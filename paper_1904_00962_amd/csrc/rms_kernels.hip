// Root-mean-square norm of rows with the residual's addition before it, its result in 8
// bits with scales, and its gradients, for gfx950.
//
//   h = x + residual, rounded to the residual's type (h = x without one)
//   y = h r w,  r = (mean(h^2) + eps)^-1/2
//   8 bits: s = max(max |y| / 448, 2^-126) over a row or a group of columns, q = e4m3(y / s)
//   backward, with g = dy w: dh = r (g - h r mean(g h r)) + ds,  dw = sum of dy h r
//
// All of it is bound by HBM: a row is read once, stays in the registers of its team's
// lanes, eight columns to a lane, and its results leave from there.
//
// Both sides of what was chosen, calls one after another in a graph, in us. Norms: bf16 to 8
// bits with a bf16 residual and groups of 128; gradients: of bf16 rows on an fp32 stream; both
// of 32768 rows of 1600 where no other size stands.
//   sums of a row in fp64 (no square passes fp32's range)  64.3, 133.4; in fp32 61.9, 132.1
//     (25000 rows: 56.9 and 51.3, the most that it costs)
//   results, but for the 8-bit ones, stored past the caches (nontemporal)  64.3, 133.4;
//     through them 73.7, 134.6
//   loads through the caches  133.4, norms of bf16 on an fp32 stream 112.8; past them 142.3,
//     117.0 (bf16 gradients of 11718 rows of 4096 gain: 77.4 and 73.3)
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

// Lanes 0 to 15 of every 16 with each other, by data-parallel moves: 1 away, 2 away, then
// eights and sixteens from their other ends. Where all lanes of a step's group hold one
// value, its mirror image is the other half's. (Shuffles, which go through LDS: 65.8 us in
// place of 64.3 for the norms above, 64.3 in place of 60.3 for 25600 rows of 3584, 4.0 in place
// of 3.7 for one row, gradients 141.6 in place of 133.4.)
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;

template <int MOVE>
__device__ inline uint32_t moved(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), MOVE, 0xF, 0xF, true));
}

template <int MOVE>
__device__ inline double moved(double v) {
    const uint64_t bits = uint64_t(__double_as_longlong(v));
    const uint32_t low = moved<MOVE>(uint32_t(bits)), high = moved<MOVE>(uint32_t(bits >> 32));
    return __longlong_as_double(int64_t(uint64_t(high) << 32 | low));
}

__device__ inline double lane_of(double v, int lane) {
    const uint64_t bits = uint64_t(__double_as_longlong(v));
    const uint32_t low = __builtin_amdgcn_readlane(uint32_t(bits), lane);
    const uint32_t high = __builtin_amdgcn_readlane(uint32_t(bits >> 32), lane);
    return __longlong_as_double(int64_t(uint64_t(high) << 32 | low));
}

// The sum over the lanes of a team (at most a wave's), on each of them. All lanes of the
// wave must be here.
template <int LANES>
__device__ inline double lanes_sum(double v) {
    v += moved<kSwap1>(v);
    v += moved<kSwap2>(v);
    v += moved<kMirror8>(v);
    v += moved<kMirror16>(v);
    if (LANES == 32)
        v += __shfl_xor(v, 16);
    if (LANES < 64)
        return v;
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// The largest of `lanes` lanes (4 to 32, a power of two) that lie together, on each of them.
__device__ inline uint32_t group_max(uint32_t v, int lanes) {
    v = max(v, moved<kSwap1>(v));
    v = max(v, moved<kSwap2>(v));
    if (lanes > 4)
        v = max(v, moved<kMirror8>(v));
    if (lanes > 8)
        v = max(v, moved<kMirror16>(v));
    if (lanes > 16)
        v = max(v, uint32_t(__shfl_xor(int(v), 16)));
    return v;
}

template <int LANES>
__device__ inline uint32_t lanes_max(uint32_t v) {
    if (LANES < 64)
        return group_max(v, LANES);
    v = group_max(v, 16);
    const uint32_t a = max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16));
    const uint32_t b = max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48));
    return max(a, b);
}

// 1 / sqrt(v) to 2^-43: the hardware's estimate (2^-22) and a Newton step, which
// makes NaN of 0 and infinity, where the estimate is right.
__device__ inline double inverse_root(double v) {
    const double y = __builtin_amdgcn_rsq(v);
    const double better = y * fma(-0.5 * v * y, y, 1.5);
    return isnan(better) ? y : better;
}

// A value that all lanes of the wave have, in a scalar register.
__device__ inline float of_wave(float v) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

// The bits of |v| as integers have the order of their values, and NaN above all.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// r as an fp32 number, and a power of two that elements take first where r is no normal one
// (all of a row within a factor of four of fp32's ends, or below them with eps 0).
struct Inverse {
    float value, shift;
    __device__ inline explicit Inverse(double r) {
        const bool small = r > 0x1p126, large = r < 0x1p-126;
        shift = small ? 0x1p64f : large ? 0x1p-64f : 1.0f;
        value = float(small ? r * 0x1p-64 : large ? r * 0x1p64 : r);
    }
    // Of a row that the whole wave has. (The wide rows' second pass needs the registers: 5300
    // fp32 rows of 9001 with a bf16 grad_x 200.7 us so, 221.5 in vector registers.)
    __device__ inline Inverse of_wave() const {
        Inverse to = *this;
        to.value = lamb_mi355x::of_wave(value);
        to.shift = lamb_mi355x::of_wave(shift);
        return to;
    }
    __device__ inline void times(float (&h)[8]) const {
        if (shift != 1.0f) {
            asm volatile("");  // stays a branch, for a whole row
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] *= shift;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= value;
    }
    // v r + add; no branch here, which would hold more registers
    __device__ inline float times_add(float v, float add) const {
        return fmaf(v * shift, value, add);
    }
};

// max(largest / 448, 2^-126) of the bits of a magnitude, and its inverse, both as if
// divided: an estimate and what it leaves. Not so for infinity and NaN.
//
// Values take the inverse, where a division would take the scale: 3 in 100000 of a bf16
// stream, whose quotients lie at ties of e4m3, then fall to the other side, no further off.
// Quotients with what the product leaves cost up to 6%: 25600 rows of 3584 60.8 us so and 64.3,
// 32768 of 1600 64.8 and 65.2; 5% more where it is below fp32's normal numbers.
__device__ inline void scale_of(uint32_t largest, float *scale, float *up) {
    const float most = __uint_as_float(largest);
    if (largest >= 0x7f800000u) {
        *scale = most;
        *up = 1.0f / most;
        return;
    }
    constexpr float kPart = 1.0f / kLargestE4m3;
    const float s = most * kPart;
    *scale = fmaxf(fmaf(fmaf(-kLargestE4m3, s, most), kPart, s), kLeastScale);
    const float u = __builtin_amdgcn_rcpf(*scale);
    *up = fmaf(fmaf(-*scale, u, 1.0f), u, u);
}

// L lanes to a row (16, 32 or whole waves), V times 8 L columns; a workgroup of one or more
// rows. With QUANT the result is 8 bits wide. TAIL: dim is no multiple of eight.
//
// One row to a team and many workgroups, not few that go from row to row: these were slower
// (112 to 118-128 us for 32768 rows of 1600, bf16 on an fp32 stream), with the next row's
// loads ahead or not. That case moves 629 MB in 110 to 112 us, 5.7 TB/s (a copy of 1 GiB
// moves 5.1); to 8 bits with groups of 128, bf16 stream: 369 MB in 61 us, 6.0 TB/s. 64 rows
// take 2.9 us, one 2.3: latency.
constexpr int rms_block(int lanes) { return lanes < kRmsBlock ? kRmsBlock : lanes; }

template <int L, int V, bool TAIL, bool X_BF16, bool RES, bool RES_BF16, bool QUANT>
__global__ __launch_bounds__(rms_block(L)) void rms_kernel(RmsArgs a, RmsOut o) {
    constexpr int kTeams = rms_block(L) / L, kWaves = L < 64 ? 1 : L / 64;
    constexpr int kInWave = L < 64 ? L : 64;
    // registers allow all loads of a row at once, and the weight's with them
    constexpr bool kTogether = V <= 4, kEarly = V <= 2;
    __shared__ double part[kTeams][kWaves];
    __shared__ uint32_t top[kTeams][kWaves];
    const int t = threadIdx.x % L, team = threadIdx.x / L, wave = t / 64;
    const int64_t row = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * kTeams + team;
    const bool live = row < a.tokens;
    int c[V], n[V];  // a lane's columns, and how many there are from there on
    Eight<X_BF16> x[V];
    Eight<RES_BF16> r[V];
    float h[V][8], w[V][8];
    auto load = [&](int v) {
        x[v] = load_eight<X_BF16, TAIL>(a.x, row * a.x_stride + c[v], n[v], c[v] > 0);
        if (RES)
            r[v] = load_eight<RES_BF16, TAIL>(a.residual, row * a.residual_stride + c[v], n[v],
                                              c[v] > 0);
    };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = (v * L + t) * 8;
        n[v] = live ? a.dim - c[v] : 0;
        if (kTogether)
            load(v);
    }
    if (kEarly && a.weight) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            load_values<TAIL>(a.weight_bf16, a.weight, c[v], a.dim - c[v], c[v] > 0, w[v]);
    }
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!kTogether)
            load(v);
        settle<TAIL>(x[v], n[v], c[v] > 0);
        x[v].get(h[v]);
        if (RES) {
            float with[8];
            settle<TAIL>(r[v], n[v], c[v] > 0);
            r[v].get(with);
#pragma unroll
            for (int i = 0; i < 8; ++i) with[i] += h[v][i];
            r[v].set(with);
            r[v].get(h[v]);
            if (o.summed)
                store_eight<RES_BF16, TAIL, true>(o.summed, row * o.summed_stride + c[v], n[v],
                                                  r[v]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma(double(h[v][i]), double(h[v][i]), sum);
    }
    sum = lanes_sum<kInWave>(sum);
    if (kWaves > 1) {
        if (t % 64 == 0)
            part[team][wave] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) sum += part[team][k];
    }
    const Inverse inverse(inverse_root(fma(sum, a.per_column, double(a.eps))));
    uint32_t largest = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        inverse.times(h[v]);
        if (a.weight) {
            if (!kEarly)
                load_values<TAIL>(a.weight_bf16, a.weight, c[v], n[v], c[v] > 0, w[v]);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] *= w[v][i];
        }
        if (!QUANT) {
            store_values<TAIL, true>(o.out_bf16, o.out, row * o.out_stride + c[v], n[v], h[v]);
        } else if (o.group == 0) {
            // columns past the row are 0 inverse, which may be NaN
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!TAIL ? n[v] > 0 : i < n[v])
                    largest = max(largest, magnitude(h[v][i]));
        }
    }
    if (!QUANT)
        return;
    if (o.group == 0) {
        largest = lanes_max<kInWave>(largest);
        if (kWaves > 1) {
            if (t % 64 == 0)
                top[team][wave] = largest;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kWaves; ++k) largest = max(largest, top[team][k]);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (o.group) {
            largest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!TAIL ? n[v] > 0 : i < n[v])
                    largest = max(largest, magnitude(h[v][i]));
            largest = group_max(largest, min(o.group / 8, kInWave));
        }
        float scale, up;
        scale_of(largest, &scale, &up);
        if (n[v] <= 0)
            continue;
        if (o.group ? c[v] % o.group == 0 : c[v] == 0)
            o.scales[row * o.groups + (o.group ? c[v] / o.group : 0)] = scale;
        uint32_t q[2] = {};
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            int word = 0;
            word = __builtin_amdgcn_cvt_pk_fp8_f32(h[v][i] * up, h[v][i + 1] * up, word, false);
            word = __builtin_amdgcn_cvt_pk_fp8_f32(h[v][i + 2] * up, h[v][i + 3] * up, word, true);
            q[i / 4] = uint32_t(word);
        }
        uint8_t *p = (uint8_t *)o.out + row * o.out_stride + c[v];
        if (n[v] >= 8) {
            __builtin_memcpy(p, q, 8);
        } else if (TAIL) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n[v])
                    p[i] = uint8_t(q[i / 4] >> (i % 4 * 8));
        }
    }
}

// Writes, or adds to, a column of the weight's gradient.
__device__ inline void finish_weight(const RmsGrad &g, int c, double sum) {
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

// A team's columns of row after row; what a lane adds to the weight's gradient stays in
// its registers, kRmsFoldRows rows to a sum and these sums to another, so that chains of like
// terms stay short. The teams' are joined at the end, and leave as one row of parts, or
// finished where there is one workgroup.
//
// Bound by HBM: 32768 rows of 1600 on an fp32 stream, 734 MB in 125 us, 5.9 TB/s; 8192 rows of
// 1024 in bf16 14 us, 4.8 TB/s. Loading the next row ahead changed neither. L = 1024 (4097 to
// 8192 columns) has 128 registers a lane, 2 to 11 fewer than the loop takes: 12 to 36 bytes a
// lane go to scratch; and one workgroup fills a CU, so that nothing loads while it joins a
// row's sums: 9600 bf16 rows of 5000 with the stream's 99 us, 3.9 TB/s, 5859 of 8192 82 us,
// 4.7. The weight loaded again for each row, in place of its registers: 6 us more for both.
template <int L, bool TAIL, bool X_BF16, bool DY_BF16, bool DX_BF16>
__global__ __launch_bounds__(L < 1024 ? 512 : 1024) void rms_grad_kernel(RmsArgs a, RmsGrad g) {
    constexpr int kWaves = L < 64 ? 1 : L / 64, kInWave = L < 64 ? L : 64;
    extern __shared__ float joined[];  // [teams][8 L], where there are teams
    __shared__ double part[2][16][2];
    const int teams = blockDim.x / L;
    const int t = threadIdx.x % L, team = threadIdx.x / L;
    const int c = t * 8, columns = a.dim - c;
    const int64_t step = int64_t(gridDim.x) * teams;
    float w[8], recent[8] = {}, dw[8] = {};
    struct Row {
        Eight<X_BF16> x;
        Eight<DY_BF16> dy;
        Eight<DX_BF16> ds;
    };
    auto load = [&](int64_t row, int n) {
        Row e;
        e.x = load_eight<X_BF16, TAIL>(a.x, row * a.x_stride + c, n, c > 0);
        e.dy = load_eight<DY_BF16, TAIL>(g.grad_out, row * g.grad_out_stride + c, n, c > 0);
        if (g.grad_sum)
            e.ds = load_eight<DX_BF16, TAIL>(g.grad_sum, row * g.grad_sum_stride + c, n, c > 0);
        else
            e.ds = Eight<DX_BF16>{};
        return e;
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.0f;
    if (a.weight)
        load_values<TAIL>(a.weight_bf16, a.weight, c, columns, c > 0, w);
    // every team of a workgroup makes as many turns
    int turn = 0;
    for (int64_t first = int64_t(blockIdx.x) * teams; first < a.tokens; first += step) {
        const int64_t row = first + team;
        const int n = row < a.tokens ? columns : 0;
        Row now = load(row, n);
        float x[8], dy[8], gw[8];
        settle<TAIL>(now.x, n, c > 0);
        settle<TAIL>(now.dy, n, c > 0);
        settle<TAIL>(now.ds, n, c > 0);
        now.x.get(x);
        now.dy.get(dy);
        double square = 0.0, along = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gw[i] = dy[i] * w[i];
            square = fma(double(x[i]), double(x[i]), square);
            along = fma(double(x[i]), double(gw[i]), along);
        }
        square = lanes_sum<kInWave>(square);
        along = lanes_sum<kInWave>(along);
        if (kWaves > 1) {
            double(*to)[2] = part[turn & 1] + threadIdx.x / L * kWaves;
            if (t % 64 == 0) {
                to[t / 64][0] = square;
                to[t / 64][1] = along;
            }
            __syncthreads();
            square = along = 0.0;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                square += to[k][0];
                along += to[k][1];
            }
        }
        const double r = inverse_root(fma(square, a.per_column, double(a.eps)));
        const Inverse inverse(r);
        const float mean = float(along * r * a.per_column);
        float ds[8], dx[8];
        now.ds.get(ds);
        if (n > 0) {
            inverse.times(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dx[i] = inverse.times_add(fmaf(-x[i], mean, gw[i]), ds[i]);
                recent[i] = fmaf(dy[i], x[i], recent[i]);
            }
            if (g.grad_x) {
                Eight<DX_BF16> e;
                e.set(dx);
                store_eight<DX_BF16, TAIL, true>(g.grad_x, row * g.grad_x_stride + c, n, e);
            }
        }
        if (++turn % kRmsFoldRows == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] += recent[i];
                recent[i] = 0.0f;
            }
        }
    }
    if (!g.grad_weight)
        return;
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] += recent[i];
    if (teams > 1) {
        // element i of lane t lies at i L + t: no two lanes of a wave in one bank
#pragma unroll
        for (int i = 0; i < 8; ++i) joined[(team * 8 + i) * L + t] = dw[i];
        __syncthreads();
        if (team > 0)
            return;
        for (int k = 1; k < teams; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[i] += joined[(k * 8 + i) * L + t];
    }
    if (gridDim.x == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < columns)
                finish_weight(g, c + i, double(dw[i]));
    } else if (columns > 0) {
        Eight<false> e;
        e.set(dw);
        store_eight<false, false>(g.partial, int64_t(blockIdx.x) * g.columns + c, 8, e);
    }
}

// Rows too wide for one lane's registers: first each row's two numbers, a workgroup a row.
// (Both passes read x and dy: 2900 bf16 rows of 16384 take 114 us, 3.3 TB/s of what has to
// move, 4.8 of what does.)
template <bool TAIL, bool X_BF16, bool DY_BF16>
__global__ __launch_bounds__(1024) void rms_stats_kernel(RmsArgs a, RmsGrad g) {
    __shared__ double part[16][2];
    const int64_t row = int64_t(blockIdx.y) * gridDim.x + blockIdx.x;
    if (row >= a.tokens)
        return;
    double square = 0.0, along = 0.0;
    for (int c = threadIdx.x * 8; c < a.dim; c += 8192) {
        const int n = a.dim - c;
        Eight<X_BF16> xe = load_eight<X_BF16, TAIL>(a.x, row * a.x_stride + c, n, c > 0);
        Eight<DY_BF16> de =
            load_eight<DY_BF16, TAIL>(g.grad_out, row * g.grad_out_stride + c, n, c > 0);
        float x[8], dy[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.0f;
        if (a.weight)
            load_values<TAIL>(a.weight_bf16, a.weight, c, n, c > 0, w);
        settle<TAIL>(xe, n, c > 0);
        settle<TAIL>(de, n, c > 0);
        xe.get(x);
        de.get(dy);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            square = fma(double(x[i]), double(x[i]), square);
            along = fma(double(x[i]), double(dy[i] * w[i]), along);
        }
    }
    square = lanes_sum<64>(square);
    along = lanes_sum<64>(along);
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
        const double r = inverse_root(fma(square, a.per_column, double(a.eps)));
        g.stats[2 * row] = r;
        g.stats[2 * row + 1] = along * r * a.per_column;
    }
}

// Then 2048 columns of kRmsWideRows rows in a workgroup, four rows in flight.
template <bool TAIL, bool X_BF16, bool DY_BF16, bool DX_BF16>
__global__ __launch_bounds__(256) void rms_wide_grad_kernel(RmsArgs a, RmsGrad g) {
    constexpr int kAhead = 4;
    const int c = (int(blockIdx.y) * 256 + threadIdx.x) * 8, columns = a.dim - c;
    if (columns <= 0)
        return;
    float w[8], dw[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.0f;
    if (a.weight)
        load_values<TAIL>(a.weight_bf16, a.weight, c, columns, c > 0, w);
    const int64_t first = int64_t(blockIdx.x) * kRmsWideRows;
    for (int64_t at = first; at < first + kRmsWideRows && at < a.tokens; at += kAhead) {
        Eight<X_BF16> xe[kAhead];
        Eight<DY_BF16> de[kAhead];
        Eight<DX_BF16> se[kAhead];
        int n[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t row = at + k;
            n[k] = row < a.tokens ? columns : 0;
            xe[k] = load_eight<X_BF16, TAIL>(a.x, row * a.x_stride + c, n[k], c > 0);
            de[k] = load_eight<DY_BF16, TAIL>(g.grad_out, row * g.grad_out_stride + c, n[k], c > 0);
            se[k] = Eight<DX_BF16>{};
            if (g.grad_sum)
                se[k] = load_eight<DX_BF16, TAIL>(g.grad_sum, row * g.grad_sum_stride + c, n[k],
                                                  c > 0);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (n[k] <= 0)
                break;
            const int64_t row = at + k;
            settle<TAIL>(xe[k], n[k], c > 0);
            settle<TAIL>(de[k], n[k], c > 0);
            settle<TAIL>(se[k], n[k], c > 0);
            float x[8], dy[8], ds[8], dx[8];
            xe[k].get(x);
            de[k].get(dy);
            se[k].get(ds);
            const Inverse inverse = Inverse(g.stats[2 * row]).of_wave();
            const float mean = of_wave(float(g.stats[2 * row + 1]));
            inverse.times(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dx[i] = inverse.times_add(fmaf(-x[i], mean, dy[i] * w[i]), ds[i]);
                dw[i] = fmaf(dy[i], x[i], dw[i]);
            }
            if (g.grad_x) {
                Eight<DX_BF16> e;
                e.set(dx);
                store_eight<DX_BF16, TAIL, true>(g.grad_x, row * g.grad_x_stride + c, n[k], e);
            }
        }
    }
    if (g.grad_weight) {
        Eight<false> e;
        e.set(dw);
        store_eight<false, false>(g.partial, int64_t(blockIdx.x) * g.columns + c, 8, e);
    }
}

// The weight's gradient: its parts in their order, 32 stripes of them and 32 columns in a
// workgroup, in fp64. 3.8 to 4.7 us for 1024 or 512 parts of 1024 and 1600 columns: latency.
__global__ __launch_bounds__(1024) void rms_join_kernel(RmsArgs a, RmsGrad g) {
    __shared__ double part[32][32];
    const int column = threadIdx.x % 32, stripe = threadIdx.x / 32;
    const int c = int(blockIdx.x) * 32 + column;
    double sum = 0.0;
    if (c < a.dim) {
#pragma unroll 16
        for (int64_t k = stripe; k < g.partials; k += 32)
            sum += double(g.partial[k * g.columns + c]);
    }
    part[stripe][column] = sum;
    __syncthreads();
    if (stripe == 0 && c < a.dim) {
        sum = 0.0;
        for (int k = 0; k < 32; ++k) sum += part[k][column];
        finish_weight(g, c, sum);
    }
}

// Lanes of a row's team: the fewest that hold it, eight columns each.
int lanes_of(int32_t dim) {
    int lanes = 16;
    while (lanes < 1024 && dim > 8 * lanes) lanes *= 2;
    return lanes;
}

template <int N>
using Constant = std::integral_constant<int, N>;

template <bool TAIL, bool X_BF16, bool RES, bool RES_BF16, bool QUANT>
hipError_t launch_rms_of(const RmsArgs &a, const RmsOut &o, hipStream_t stream) {
    auto run = [&](auto lanes, auto times) {
        constexpr int L = decltype(lanes)::value, V = decltype(times)::value;
        constexpr int kTeams = rms_block(L) / L;
        rms_kernel<L, V, TAIL, X_BF16, RES, RES_BF16, QUANT>
            <<<grid_of((a.tokens + kTeams - 1) / kTeams), rms_block(L), 0, stream>>>(a, o);
        return hipGetLastError();
    };
    const int lanes = lanes_of(a.dim);
    // Half the lanes with twice the columns, where rows are many, a team's last lanes have no
    // columns and a lane has little to load: a wave's fixed work counts more there. 25000 rows
    // of 1600 to 8 bits 56.9 us so and 61.9 the other way, 2100 rows 9.1 and 8.7; 15625 bf16 rows
    // of 2560 without a residual 28.6 and 33.0 (fp32 63.0 and 61.4). But with one 56.9 and 54.2,
    // 2048 columns to 8 bits 48.1 and 46.2, and 64 rows of 1600 3.7 and 3.0.
    if constexpr (!TAIL && (QUANT || !RES)) {
        if (a.tokens >= 2048 && 8 * a.dim <= 7 * 8 * lanes) {
            switch (lanes) {
            case 128: return run(Constant<64>{}, Constant<2>{});
            case 256: return run(Constant<128>{}, Constant<2>{});
            case 512: return run(Constant<256>{}, Constant<2>{});
            case 1024: return run(Constant<512>{}, Constant<2>{});
            }
        }
    }
    switch (lanes) {
    case 16: return run(Constant<16>{}, Constant<1>{});
    case 32: return run(Constant<32>{}, Constant<1>{});
    case 64: return run(Constant<64>{}, Constant<1>{});
    case 128: return run(Constant<128>{}, Constant<1>{});
    case 256: return run(Constant<256>{}, Constant<1>{});
    case 512: return run(Constant<512>{}, Constant<1>{});
    }
    if (a.dim <= 8192)
        return run(Constant<1024>{}, Constant<1>{});
    if (a.dim <= 16384)
        return run(Constant<1024>{}, Constant<2>{});
    return a.dim <= 32768 ? run(Constant<1024>{}, Constant<4>{})
                          : run(Constant<1024>{}, Constant<8>{});
}

template <bool TAIL, bool QUANT>
hipError_t launch_rms_types(const RmsArgs &a, const RmsOut &o, hipStream_t stream) {
    if (!a.residual)
        return a.x_bf16 ? launch_rms_of<TAIL, true, false, true, QUANT>(a, o, stream)
                        : launch_rms_of<TAIL, false, false, false, QUANT>(a, o, stream);
    if (!a.x_bf16)
        return launch_rms_of<TAIL, false, true, false, QUANT>(a, o, stream);
    return a.residual_bf16 ? launch_rms_of<TAIL, true, true, true, QUANT>(a, o, stream)
                           : launch_rms_of<TAIL, true, true, false, QUANT>(a, o, stream);
}

template <bool TAIL>
hipError_t launch_rms_tail(const RmsArgs &a, const RmsOut &o, hipStream_t stream) {
    return o.scales ? launch_rms_types<TAIL, true>(a, o, stream)
                    : launch_rms_types<TAIL, false>(a, o, stream);
}

struct GradShape {
    int lanes, block;
    int64_t blocks;
};

// `row_bytes`: what a row reads. Few rows go to one workgroup, which needs no second launch.
// Else at least two rows each (a part of the weight's gradient for every row costs more), in
// 1024 workgroups where a turn of one reads less than 14 KB, else in 512: with more in flight
// HBM falls behind. The border lies between what was measured on its sides, 32768 rows of
// 1600 on an fp32 stream (16 KB) 133.6 us with 512 and 149.9 with 1024, 30000 of bf16 (9.6 KB)
// 96.0 and 77.6; ragged rows want more further up (192000 fp32 rows of 250, 24 KB: 175 and 149).
GradShape grad_shape(int64_t tokens, int32_t dim, int64_t row_bytes) {
    GradShape s;
    s.lanes = lanes_of(dim);
    s.block = rms_block(s.lanes);
    const int64_t few = std::max(512, s.lanes) / s.lanes;
    if (tokens <= 2 * few) {
        s.block = std::max(512, s.lanes);
        s.blocks = 1;
        return s;
    }
    const int64_t teams = s.block / s.lanes, turns = (tokens + teams - 1) / teams;
    const int64_t most = s.lanes == 1024 ? 256 : teams * row_bytes < 14336 ? 1024 : 512;
    s.blocks = std::min((turns + 1) / 2, most);
    return s;
}

int64_t row_bytes(const RmsArgs &a, const RmsGrad &g) {
    const int64_t x = a.x_bf16 ? 2 : 4, dy = g.grad_out_bf16 ? 2 : 4, ds = g.grad_x_bf16 ? 2 : 4;
    return a.dim * (x + dy + (g.grad_sum ? ds : 0));
}

template <bool TAIL, bool X_BF16, bool DY_BF16, bool DX_BF16>
hipError_t launch_wide_grad_of(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    rms_stats_kernel<TAIL, X_BF16, DY_BF16><<<grid_of(a.tokens), 1024, 0, stream>>>(a, g);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    const dim3 grid(uint32_t(g.partials), uint32_t((a.dim + 2047) / 2048));
    rms_wide_grad_kernel<TAIL, X_BF16, DY_BF16, DX_BF16><<<grid, 256, 0, stream>>>(a, g);
    return hipGetLastError();
}

template <bool TAIL, bool X_BF16, bool DY_BF16, bool DX_BF16>
hipError_t launch_rms_grad_of(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    if (a.dim > kRmsHeldDim)
        return launch_wide_grad_of<TAIL, X_BF16, DY_BF16, DX_BF16>(a, g, stream);
    const GradShape s = grad_shape(a.tokens, a.dim, row_bytes(a, g));
    auto run = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const size_t lds = s.block > L && g.grad_weight ? size_t(s.block) * 8 * 4 : 0;
        rms_grad_kernel<L, TAIL, X_BF16, DY_BF16, DX_BF16>
            <<<uint32_t(s.blocks), s.block, lds, stream>>>(a, g);
        return hipGetLastError();
    };
    switch (s.lanes) {
    case 16: return run(Constant<16>{});
    case 32: return run(Constant<32>{});
    case 64: return run(Constant<64>{});
    case 128: return run(Constant<128>{});
    case 256: return run(Constant<256>{});
    case 512: return run(Constant<512>{});
    default: return run(Constant<1024>{});
    }
}

template <bool TAIL>
hipError_t launch_rms_grad_types(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    auto by_dx = [&](auto x, auto dy) {
        constexpr bool X = decltype(x)::value, DY = decltype(dy)::value;
        return g.grad_x_bf16 ? launch_rms_grad_of<TAIL, X, DY, true>(a, g, stream)
                             : launch_rms_grad_of<TAIL, X, DY, false>(a, g, stream);
    };
    auto by_dy = [&](auto x) {
        return g.grad_out_bf16 ? by_dx(x, std::true_type{}) : by_dx(x, std::false_type{});
    };
    return a.x_bf16 ? by_dy(std::true_type{}) : by_dy(std::false_type{});
}

}  // namespace

hipError_t launch_rms(const RmsArgs &args, const RmsOut &out, hipStream_t stream) {
    return args.dim % 8 ? launch_rms_tail<true>(args, out, stream)
                        : launch_rms_tail<false>(args, out, stream);
}

int64_t rms_partials(const RmsArgs &a, const RmsGrad &g) {
    if (a.dim > kRmsHeldDim)
        return (a.tokens + kRmsWideRows - 1) / kRmsWideRows;
    return a.tokens ? grad_shape(a.tokens, a.dim, row_bytes(a, g)).blocks : 0;
}

int64_t rms_most_partials(int64_t tokens, int32_t dim) {
    if (dim > kRmsHeldDim)
        return (tokens + kRmsWideRows - 1) / kRmsWideRows;
    return tokens ? grad_shape(tokens, dim, 0).blocks : 0;  // the fewer bytes, the more
}

hipError_t launch_rms_grad(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    return a.dim % 8 ? launch_rms_grad_types<true>(a, g, stream)
                     : launch_rms_grad_types<false>(a, g, stream);
}

hipError_t launch_rms_join(const RmsArgs &a, const RmsGrad &g, hipStream_t stream) {
    if (a.dim <= kRmsHeldDim && g.partials == 1)
        return hipSuccess;  // its workgroup has done it
    rms_join_kernel<<<uint32_t((a.dim + 31) / 32), 1024, 0, stream>>>(a, g);
    return hipGetLastError();
}

}  // namespace lamb_mi355x
