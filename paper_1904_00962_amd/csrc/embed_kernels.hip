// Lookup of a token table's rows, and the table's gradient, for gfx950.
//
// The gradient of row v is the sum of the gradients of the tokens with id v, in the
// tokens' order, in fp32: the tokens are sorted by id first, so that no two sums meet
// in one address and every call gives the same bits.
//
// Sorting takes one launch. Each workgroup owns a range of ids and reads all ids twice:
// once to count its own (per wave's share of the tokens) and the smaller ones, which
// gives every id its place, and once to put its tokens there. The ids are read from L2,
// up to 8192 of them only once: with many, tokens x vocab / 512 readings.
//
// Summing cuts the sorted order, not the table, into equal chunks, so that the rows of a
// frequent id (or a batch of padding) are read by many waves. An id's tokens that lie
// within a chunk are summed and written; what reaches over a chunk's ends goes to a
// partial sum, and a second pass joins these, an id's in one wave. Rows without tokens are
// written as zeros by the first pass, unless the gradient is added to what is there.
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "embed_internal.h"
#include "ops_host.h"

namespace lamb_mi355x {
namespace {

__device__ inline uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, __bf16(v)); }
__device__ inline float widen(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }

__device__ inline int64_t id_at(const EmbedArgs &a, int64_t i) {
    return a.wide ? ((const int64_t *)a.ids)[i] : int64_t(((const int32_t *)a.ids)[i]);
}

// Eight elements from column c of a row, `n` of them inside it.
template <bool BF16>
__device__ inline void load8(const void *base, int64_t at, int n, bool vector, float (&v)[8]) {
    if (BF16) {
        const uint16_t *p = (const uint16_t *)base + at;
        if (vector && n >= 8) {
            const uint4 w = *(const uint4 *)p;
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(u[i] << 16);
                v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? widen(p[i]) : 0.0f;
    } else {
        const float *p = (const float *)base + at;
        if (vector && n >= 8) {
            const float4 lo = *(const float4 *)p, hi = *(const float4 *)(p + 4);
            v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
            v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
    }
}

template <bool BF16>
__device__ inline void store8(void *base, int64_t at, int n, bool vector, const float (&v)[8]) {
    if (BF16) {
        uint16_t *p = (uint16_t *)base + at;
        if (vector && n >= 8) {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                u[i] = uint32_t(to_bf16(v[2 * i])) | uint32_t(to_bf16(v[2 * i + 1])) << 16;
            *(uint4 *)p = make_uint4(u[0], u[1], u[2], u[3]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n)
                p[i] = to_bf16(v[i]);
    } else {
        float *p = (float *)base + at;
        if (vector && n >= 8) {
            *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
            *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n)
                p[i] = v[i];
    }
}

// Eight columns a thread. Few tokens are bound by latency: 2.7 us for 64 of 1600 columns.
template <bool TABLE_BF16, bool OUT_BF16>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, EmbedRows r) {
    const uint32_t per_row = uint32_t(a.dim + 7) / 8;
    const int64_t unit =
        (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    const int64_t units = a.tokens * per_row;
    if (unit >= units)
        return;
    const int64_t token = units <= INT32_MAX ? int64_t(uint32_t(unit) / per_row) : unit / per_row;
    const int c = int(unit - token * per_row) * 8;
    const int n = a.dim - c;
    const int64_t id = id_at(a, token);
    float v[8];
    if (id >= 0 && id < a.vocab) {
        load8<TABLE_BF16>(r.table, id * r.table_stride + c, n, r.vector, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= a.scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = NAN;
    }
    store8<OUT_BF16>(r.out, token * r.out_stride + c, n, r.vector, v);
}

// Bound by latency (two passes over LDS and L2, a scan): 9 to 11 us for 8192 tokens and
// 30522 or 50257 ids.
__global__ __launch_bounds__(kSortWaves * 64) void embed_sort_kernel(EmbedArgs a, int32_t ids,
                                                                     int64_t skip, int32_t *order,
                                                                     int32_t *sorted,
                                                                     int32_t *first) {
    extern __shared__ int32_t counts[];  // [kSortWaves][ids], then two rows of kSortWaves
    int32_t *smaller = counts + kSortWaves * ids, *group_total = smaller + kSortWaves;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t low = int64_t(blockIdx.x) * ids;
    for (int i = threadIdx.x; i < kSortWaves * ids; i += kSortWaves * 64) counts[i] = 0;
    // this wave's share of the tokens, whole groups of 64
    const int64_t groups = (a.tokens + 63) / 64;
    const int64_t share = (groups + kSortWaves - 1) / kSortWaves * 64;
    const int64_t begin = wave * share;
    const int64_t end = begin + share < a.tokens ? begin + share : a.tokens;
    constexpr int kAhead = 8;  // groups of 64 ids in flight
    int32_t *mine = counts + wave * ids;
    // the ids from token g on, less `low`: below 0 the smaller ones, kLeftOut those that
    // do not count
    constexpr int32_t kLeftOut = INT32_MAX;
    auto read = [&](int64_t g, int32_t (&local)[kAhead]) {
        int64_t id[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t i = g + 64 * k + lane;
            id[k] = i < end ? id_at(a, i) : -1;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            local[k] = id[k] == skip || id[k] < 0 || id[k] >= a.vocab ? kLeftOut
                                                                       : int32_t(id[k] - low);
    };
    int32_t held[kAhead];  // the first groups, for the second reading
    read(begin, held);
    __syncthreads();
    int32_t before = 0;
    auto count = [&](const int32_t (&local)[kAhead]) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            before += local[k] < 0;
            if (local[k] >= 0 && local[k] < ids)
                atomicAdd(&mine[local[k]], 1);
        }
    };
    count(held);
    for (int64_t g = begin + 64 * kAhead; g < end; g += 64 * kAhead) {
        int32_t local[kAhead];
        read(g, local);
        count(local);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
    if (lane == 0)
        smaller[wave] = before;
    __syncthreads();
    // every (id, wave)'s first place: a scan over the ids, 64 of them to a wave
    const int id = wave * 64 + lane;
    int32_t n[kSortWaves], total = 0, scan = 0;
    if (wave * 64 < ids) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            n[w] = counts[w * ids + id];
            total += n[w];
        }
        scan = total;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t up = __shfl_up(scan, d);
            scan += lane >= d ? up : 0;
        }
        if (lane == 63)
            group_total[wave] = scan;
    }
    __syncthreads();
    if (wave * 64 < ids) {
        int32_t place = scan - total;
        for (int w = 0; w < kSortWaves; ++w) place += smaller[w];
        for (int g = 0; g < wave; ++g) place += group_total[g];
        if (low + id < a.vocab)
            first[low + id] = place;
        if (low + id == a.vocab - 1)
            first[a.vocab] = place + total;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            counts[w * ids + id] = place;
            place += n[w];
        }
    }
    __syncthreads();
    // Put the tokens in their places, those of one id in lane order: the lanes with the
    // same id are those whose id agrees in every bit.
    const int bits = 32 - __clz(ids - 1);
    auto put = [&](int64_t g, const int32_t (&local)[kAhead]) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool inside = local[k] >= 0 && local[k] < ids;
            uint64_t same = __ballot(inside);
            if (!same)
                continue;
            for (int b = 0; b < bits; ++b) {
                const bool set = local[k] >> b & 1;
                const uint64_t with = __ballot(set);
                same &= set ? with : ~with;
            }
            if (inside) {
                const int32_t place = mine[local[k]];
                const int32_t ahead = __popcll(same & ((uint64_t(1) << lane) - 1));
                order[place + ahead] = int32_t(g + 64 * k + lane);
                sorted[place + ahead] = int32_t(low) + local[k];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                if (ahead == 0)
                    mine[local[k]] = place + __popcll(same);
            }
            // the next reader of a place may be another lane
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    };
    put(begin, held);
    for (int64_t g = begin + 64 * kAhead; g < end; g += 64 * kAhead) {
        int32_t local[kAhead];
        read(g, local);
        put(g, local);
    }
}

// Writes, or adds to `old`, a finished row's eight columns.
template <bool BF16, bool ADD>
__device__ inline void finish(const EmbedArgs &a, const EmbedGrad &g, int64_t id, int c,
                              float (&v)[8], const float (&old)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = ADD ? v[i] * a.scale + old[i] : v[i] * a.scale;
    store8<BF16>(g.table, id * g.table_stride + c, a.dim - c, g.vector, v);
}

// Waves of the first `chunks` x (columns / kSumColumns) sum a chunk's columns; where the
// gradient is not added, the waves after them write the rows without tokens. Bound by
// writing where it writes the whole table: 8192 bf16 rows of 1024 into 30522 fp32 ones take
// 22 us, 6.4 TB/s, in runs that follow one another, whose table the last-level cache holds
// in part (a fill of 4 GiB writes 6.9 TB/s, a copy of 1 GiB moves 5.1); 23.4 us where ADD was
// no template argument, as the old rows hold 64 registers. Added to 50257 bf16 rows of 1600, 18.7 us, 2.6 TB/s: latency, few rows are touched.
template <bool ROWS_BF16, bool TABLE_BF16, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, EmbedGrad g) {
    const int lane = threadIdx.x & 63;
    const int across = g.columns / kSumColumns;
    const int64_t chunks = (a.tokens + kSumTokens - 1) / kSumTokens;
    int64_t work = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (work >= chunks * across) {
        // kZeroRows rows: which of them are empty, then those one after another
        const int64_t row0 = (work - chunks * across) * kZeroRows;
        if (ADD || row0 >= a.vocab)
            return;
        const int64_t row = row0 + (lane < kZeroRows ? lane : kZeroRows);
        const int32_t from = g.first[row < a.vocab ? row : a.vocab];
        const int32_t to = __shfl_down(from, 1);
        uint64_t empty = __ballot(lane < kZeroRows && row < a.vocab && from == to);
        using T = typename std::conditional<TABLE_BF16, uint16_t, float>::type;
        constexpr int kEach = 16 / sizeof(T);
        const int whole = g.vector ? a.dim / kEach * kEach : 0;  // in 16 bytes a lane
        while (empty) {
            const int r = __ffsll((unsigned long long)empty) - 1;
            empty &= empty - 1;
            T *to = (T *)g.table + (row0 + r) * g.table_stride;
            for (int c = lane * kEach; c < whole; c += 64 * kEach)
                *(uint4 *)(to + c) = make_uint4(0, 0, 0, 0);
            for (int c = whole + lane; c < a.dim; c += 64) to[c] = T(0);
        }
        return;
    }
    const int64_t chunk = work / across;
    const int c = int(work % across) * kSumColumns + lane * 8;
    const int32_t total = g.first[a.vocab];
    const int32_t begin = int32_t(chunk) * kSumTokens;
    const int32_t end = begin + kSumTokens < total ? begin + kSumTokens : total;
    if (begin >= total)
        return;
    // lane t holds the chunk's t-th token and id
    const int32_t at = begin + lane < end ? begin + lane : end - 1;
    const int32_t token_of = g.order[at], id_of = g.sorted[at];
    const int n = a.dim - c;
    const int32_t id_before = begin > 0 ? g.sorted[begin - 1] : -1;
    const int32_t id_after = end < total ? g.sorted[end] : -1;
    float sum[8] = {};
    // rows in flight, and with them what the table holds for the ids that end there
    constexpr int kAhead = 8;
    for (int t0 = 0; t0 < end - begin; t0 += kAhead) {
        float row[kAhead][8], old[kAhead][8];
        int32_t id[kAhead];
        bool ends[kAhead], whole[kAhead];  // the id's last token here; all of them are here
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int t = t0 + k;
            const int32_t token = __shfl(token_of, t);
            id[k] = __shfl(id_of, t);
            const bool last = t + 1 == end - begin;
            const int32_t after = last ? id_after : __shfl(id_of, t + 1);
            ends[k] = last || after != id[k];
            whole[k] = ends[k] && after != id[k] && id[k] != id_before;
            if (t < end - begin && n > 0) {
                load8<ROWS_BF16>(g.rows, token * g.rows_stride + c, n, g.vector, row[k]);
                if (ADD && whole[k])
                    load8<TABLE_BF16>(g.table, id[k] * g.table_stride + c, n, g.vector, old[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (t0 + k >= end - begin)
                break;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += row[k][i];
            if (!ends[k])
                continue;
            if (n > 0) {
                if (whole[k]) {
                    finish<TABLE_BF16, ADD>(a, g, id[k], c, sum, old[k]);
                } else {
                    // an id that reaches back goes to the chunk's first slot, one that
                    // only reaches on to its second
                    float *to = g.partial + (2 * chunk + (id[k] != id_before)) * g.columns + c;
                    *(float4 *)to = make_float4(sum[0], sum[1], sum[2], sum[3]);
                    *(float4 *)(to + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
        }
    }
}

// A wave per chunk and kSumColumns columns: if an id begins in the chunk and goes on,
// its partial sums from there on, in order, kJoinChunks at a time. Bound by latency: 5 us
// for 8192 tokens of text. An id that holds all tokens is one wave's for each kSumColumns
// columns, with a partial sum for every 16 tokens: calls of 2^17 and 2^20 tokens of 64
// columns take 0.70 and 5.5 ms so, 0.10 and 0.83 where the ids are spread over 50257.
template <bool TABLE_BF16, bool ADD>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a, EmbedGrad g) {
    const int lane = threadIdx.x & 63;
    const int across = g.columns / kSumColumns;
    const int64_t work = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int64_t chunk = work / across;
    const int c = int(work % across) * kSumColumns + lane * 8;
    const int32_t total = g.first[a.vocab];
    const int64_t end = (chunk + 1) * kSumTokens;
    if (end >= total || c >= a.dim)
        return;
    const int32_t id = g.sorted[end - 1];
    if (g.sorted[end] != id || g.first[id] < chunk * kSumTokens)
        return;
    const int64_t last = (g.first[id + 1] - 1) / kSumTokens;
    float sum[8], old[8] = {};
    if (ADD)
        load8<TABLE_BF16>(g.table, id * g.table_stride + c, a.dim - c, g.vector, old);
    load8<false>(g.partial, (2 * chunk + 1) * g.columns + c, 8, true, sum);
    for (int64_t k0 = chunk + 1; k0 <= last; k0 += kJoinChunks) {
        const int64_t end = k0 + kJoinChunks <= last ? k0 + kJoinChunks : last + 1;
        float part[8], group[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) group[i] = k0 == chunk + 1 ? sum[i] : 0.0f;
#pragma unroll 8
        for (int64_t k = k0; k < end; ++k) {
            load8<false>(g.partial, 2 * k * g.columns + c, 8, true, part);
#pragma unroll
            for (int i = 0; i < 8; ++i) group[i] += part[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = k0 == chunk + 1 ? group[i] : sum[i] + group[i];
    }
    finish<TABLE_BF16, ADD>(a, g, id, c, sum, old);
}

}  // namespace

hipError_t launch_embed(const EmbedArgs &args, const EmbedRows &rows, hipStream_t stream) {
    const int64_t units = args.tokens * ((args.dim + 7) / 8);
    auto kernel = rows.table_bf16
                      ? (rows.out_bf16 ? embed_kernel<true, true> : embed_kernel<true, false>)
                      : (rows.out_bf16 ? embed_kernel<false, true> : embed_kernel<false, false>);
    kernel<<<grid_of((units + 255) / 256), 256, 0, stream>>>(args, rows);
    return hipGetLastError();
}

hipError_t launch_embed_sort(const EmbedArgs &args, int64_t skip, int32_t *order, int32_t *sorted,
                             int32_t *first, hipStream_t stream) {
    const int32_t ids = sort_ids(args.tokens);
    const uint32_t blocks = uint32_t((args.vocab + ids - 1) / ids);
    embed_sort_kernel<<<blocks, kSortWaves * 64, (ids + 2) * kSortWaves * 4, stream>>>(
        args, ids, skip, order, sorted, first);
    return hipGetLastError();
}

hipError_t launch_embed_sum(const EmbedArgs &args, const EmbedGrad &grad, hipStream_t stream) {
    const int64_t chunks = (args.tokens + kSumTokens - 1) / kSumTokens;
    const int64_t zeros = grad.add ? 0 : (args.vocab + kZeroRows - 1) / kZeroRows;
    const int64_t waves = chunks * (grad.columns / kSumColumns) + zeros;
    auto pick = [&](auto add) {
        constexpr bool A = decltype(add)::value;
        return grad.rows_bf16
                   ? (grad.table_bf16 ? embed_sum_kernel<true, true, A>
                                      : embed_sum_kernel<true, false, A>)
                   : (grad.table_bf16 ? embed_sum_kernel<false, true, A>
                                      : embed_sum_kernel<false, false, A>);
    };
    auto kernel = grad.add ? pick(std::true_type{}) : pick(std::false_type{});
    kernel<<<uint32_t((waves + 3) / 4), 256, 0, stream>>>(args, grad);
    return hipGetLastError();
}

hipError_t launch_embed_join(const EmbedArgs &args, const EmbedGrad &grad, hipStream_t stream) {
    const int64_t chunks = (args.tokens + kSumTokens - 1) / kSumTokens;
    const int64_t waves = chunks * (grad.columns / kSumColumns);
    auto kernel = grad.table_bf16
                      ? (grad.add ? embed_join_kernel<true, true> : embed_join_kernel<true, false>)
                      : (grad.add ? embed_join_kernel<false, true>
                                  : embed_join_kernel<false, false>);
    kernel<<<uint32_t((waves + 3) / 4), 256, 0, stream>>>(args, grad);
    return hipGetLastError();
}

}  // namespace lamb_mi355x
