// A workgroup's tile of a matrix product D = A B^T on the matrix cores, from
// 16-bit operands into fp32 accumulators. Device code shared by the kernels of
// the Newton-Schulz products and of the cross entropy. Not installed.
//
// Each operand is one of two kinds, so that no kernel needs a transposed copy:
//  rows     its rows are D's rows (or columns) and the summed index k runs along
//           a row: element (i, k) at i * ld + k
//  columns  its rows are k: element (i, k) at k * ld + i
// LDS holds a ring of stages, each some values of k of both operands; the loads of
// all but one run while that one is computed on. Global memory goes
// there directly (16 bytes a lane), so no register holds data in flight; what
// lies outside an operand is given an offset past the buffer's length, which the
// load unit answers with zeros.
//
// LDS is written in lane order, so the order of a stage is set by which 16-byte
// piece each lane asks for. Pieces are swapped within a row (rows: row_slot) or in
// pairs (columns: column_slot) such that the lanes served together in a fragment
// read touch every bank once.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace lamb_mi355x {

using half8 = _Float16 __attribute__((ext_vector_type(8)));
using bf8 = __bf16 __attribute__((ext_vector_type(8)));
using short4v = short __attribute__((ext_vector_type(4)));
using short8v = short __attribute__((ext_vector_type(8)));
using float4v = float __attribute__((ext_vector_type(4)));
using int4v = int __attribute__((ext_vector_type(4)));

constexpr int kBufferWord3 = 0x00027000;  // raw 32-bit buffer, gfx9
constexpr int kBufferBytes = 0x7ffffff0;  // a voffset with the sign bit set is outside
constexpr int kOutside = int(0x80000000u);

#define LAMB_LDS __attribute__((address_space(3)))
#define LAMB_GLOBAL __attribute__((address_space(1)))

template <int BYTES>
struct Words {
    using Type = uint32_t __attribute__((ext_vector_type(BYTES / 4)));
};
template <>
struct Words<4> {
    using Type = uint32_t;
};
template <>
struct Words<2> {
    using Type = uint16_t;
};

// Global memory through pointers that themselves come out of memory, which the
// compiler would else access as possibly LDS.
template <class T>
__device__ inline T load_global(const void *p) {
    const auto w = *(LAMB_GLOBAL const typename Words<sizeof(T)>::Type *)p;
    T v;
    __builtin_memcpy(&v, &w, sizeof v);
    return v;
}
template <class T>
__device__ inline void store_global(void *p, T v) {
    typename Words<sizeof(T)>::Type w;
    __builtin_memcpy(&w, &v, sizeof v);
    *(LAMB_GLOBAL typename Words<sizeof(T)>::Type *)p = w;
}

struct HalfMath {
    using Elem = _Float16;
    static __device__ float4v mma(short8v a, short8v b, float4v c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                      __builtin_bit_cast(half8, b), c, 0, 0, 0);
    }
};

struct Bf16Math {
    using Elem = __bf16;
    static __device__ float4v mma(short8v a, short8v b, float4v c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a),
                                                       __builtin_bit_cast(bf8, b), c, 0, 0, 0);
    }
};

// An operand of one tile: `base` at the tile's first row (rows) or column
// (columns) and k = 0, `ld` in bytes, `extent` the rows or columns from there on
// that exist (columns: in multiples of 8).
struct Operand {
    const char *base;
    int64_t ld;
    int32_t extent;
};

// Tile shape: BM x BN by WM x WN waves of 64, STAGES stages of DEPTH values of k
// each; PARTS 2 for operands that are each the sum of two parts.
template <int BM_, int BN_, int WM_, int WN_, int DEPTH_, int STAGES_, int PARTS_>
struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int DEPTH = DEPTH_, STAGES = STAGES_, PARTS = PARTS_;
    static constexpr int kWaves = WM * WN;
    static constexpr int kThreads = kWaves * 64;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int kA = BM * DEPTH, kB = BN * DEPTH;  // a part's 16-bit elements
    static constexpr int kStage = (kA + kB) * PARTS;
    static constexpr int kLds = kStage * STAGES;
    static constexpr int kLoads = kStage / 8 / kThreads;  // a lane's loads per stage
    // small tiles have too few matrix instructions a phase to pay for its meetings
    static constexpr bool kAlternating = BM == 256;
    // workgroups per CU: what LDS allows, and at most two
    static constexpr int kPerCu = 160 * 1024 / (kLds * 2) >= 2 ? 2 : 1;
    static_assert(DEPTH % 32 == 0 && STAGES >= 2 && kLds * 2 <= 160 * 1024 &&
                      kLoads * (STAGES - 2) < 64,
                  "");
};

// Bank swizzle of a `rows` stage: 8 rows at the same k get different banks.
template <int DEPTH>
__device__ inline int row_slot(int row) {
    return DEPTH == 64 ? row & 7 : (row >> 1) & 3;
}

// Bank swizzle of a `columns` stage: rows of k that one fragment read touches
// (8 q + j, q = 0, 1 together, j = 0..3) get different slots.
__device__ inline int column_slot(int k) { return (k & 3) | ((k >> 1) & 4); }

// `v`, the same on every lane, in a scalar register that a scalar instruction wrote. A
// vector instruction's scalar result must not be read by a load within 5 wait states;
// the compiler sees to that for its own loads, but not for load_to_lds.
__device__ inline int scalar(int v) {
    int s;
    asm volatile("s_mov_b32 %0, %1" : "=s"(s) : "s"(__builtin_amdgcn_readfirstlane(v)));
    return s;
}

// 16 bytes a lane from rsrc + off to LDS at `lds` + 16 lane; rsrc's words and lds have
// been through scalar(). The builtin for this makes the compiler wait for every load
// in flight before the next LDS read, which would end the overlap of a stage's loads
// with the stage before; written out, the waiting is tile_product's. The load has no
// register result, so nothing can be reused under it. (M0 needs one wait state.)
__device__ inline void load_to_lds(int4v rsrc, int off, int lds) {
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(off), "s"(rsrc), "{m0}"(lds));
}

// One operand's share of a stage: EXT rows (or columns) by DEPTH.
template <int EXT, int DEPTH, int WAVES, bool COLUMNS>
struct StageLoader {
    static constexpr int kLoads = EXT * DEPTH / 8 / 64 / WAVES;
    static_assert(kLoads >= 1 && kLoads * 512 * WAVES == EXT * DEPTH, "whole waves of 16 bytes");
    static constexpr int kPieces = COLUMNS ? EXT / 8 : DEPTH / 8;  // 16-byte pieces of a stage row
    static constexpr int kSlots = EXT / 16 < 8 ? EXT / 16 - 1 : 7;  // columns: swap within these
    static constexpr int kNext = COLUMNS ? 64 / kPieces : 0;  // k from one load to the next
    int offset[kLoads];  // from the operand's base at the stage's first k
    int first_k;         // the lane's k in the stage, of its first load

    __device__ void init(const Operand &op, int wave, int lane) {
#pragma unroll
        for (int t = 0; t < kLoads; ++t) {
            const int at = (wave * kLoads + t) * 64 + lane;  // piece of the stage
            const int row = at / kPieces, p = at % kPieces;
            if (COLUMNS) {
                const int col = ((((p >> 1) ^ (column_slot(row) & kSlots)) << 1) | (p & 1)) * 8;
                offset[t] = col < op.extent ? int(row * op.ld) + col * 2 : kOutside;
                if (t == 0)
                    first_k = row;
            } else {
                const int k = (p ^ row_slot<DEPTH>(row)) * 8;
                offset[t] = row < op.extent ? int(row * op.ld) + k * 2 : kOutside;
                if (t == 0)
                    first_k = k;  // the same of every load: rows 64 / kPieces apart
            }
        }
    }

    // `src` at the stage's first k, of which `left` remain (none or less: zeros).
    __device__ void issue(const char *src, int64_t left, const short *stage, int wave) const {
        const uint64_t at = reinterpret_cast<uint64_t>(src);
        const int4v rsrc = {scalar(int(at)), scalar(int(at >> 32) & 0xffff), kBufferBytes,
                            kBufferWord3};
        const int lds =
            scalar(int(uintptr_t((LAMB_LDS const short *)stage)) + wave * kLoads * 1024);
        const bool whole = left >= DEPTH;
#pragma unroll
        for (int t = 0; t < kLoads; ++t) {
            const int off = whole || first_k + t * kNext < left ? offset[t] : kOutside;
            load_to_lds(rsrc, off, lds + t * 1024);
        }
    }
};

// The fragment of rows first .. first + 15 for k = 32 step + 8 (lane / 16) + 0..7.
template <int EXT, int DEPTH, bool COLUMNS>
__device__ inline short8v read_fragment(const short *stage, int first, int step, int lane) {
    if (COLUMNS) {
        constexpr int kSlots = EXT / 16 < 8 ? EXT / 16 - 1 : 7;
        const int k = step * 32 + (lane >> 4) * 8 + ((lane >> 2) & 3);
        short8v both;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int kk = k + 4 * h;
            const int pair = (first >> 4) ^ (column_slot(kk) & kSlots);
            const short4v v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (LAMB_LDS short4v *)(stage + kk * EXT + pair * 16 + (lane & 3) * 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) both[4 * h + j] = v[j];
        }
        return both;
    }
    const int row = first + (lane & 15);
    const int piece = (step * 4 + (lane >> 4)) ^ row_slot<DEPTH>(row);
    return *(const short8v *)(stage + row * DEPTH + piece * 8);
}

// Before a stage is read its loads have landed (every wave waits for its own, of
// which OPEN later ones may still run, then all meet); the same meeting says that the
// stage before has been read. The stages' addresses went to the loads, so the
// compiler takes them as written here.
template <int OPEN>
__device__ inline void meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(OPEN) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Computes on stages 0 .. count - 1. issue(stage) starts the next one's loads (zeros
// past the end, so that every turn has the same number of loads in flight). On
// return no load runs and all of LDS may be written.
template <class Shape, class Issue, class Compute>
__device__ inline void run_stages(int32_t count, const short *lds, Issue issue, Compute compute) {
#pragma unroll
    for (int s = 0; s < Shape::STAGES - 1; ++s) issue(lds + s * Shape::kStage);
    const short *reads = lds, *writes = lds + (Shape::STAGES - 1) * Shape::kStage;
    const short *end = lds + Shape::kLds;
    auto next = [&](const short *p) {
        p += Shape::kStage;
        return p == end ? lds : p;
    };
    for (int32_t it = 0; it < count; ++it) {
        meet<(Shape::STAGES - 2) * Shape::kLoads>();
        issue(writes);
        compute(reads);
        reads = next(reads);
        writes = next(writes);
    }
    meet<0>();
}

// A meeting in the middle of a turn: what has been read from LDS is in registers, and
// OPEN of the wave's loads may still run. Nothing moves over it.
template <int OPEN>
__device__ inline void phase() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(OPEN) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The alternating form, for workgroups of 8 waves that have a CU to themselves. The
// waves 0..3 and 4..7 are a phase apart, so that of the two waves on a SIMD one reads
// fragments while the other's matrix instructions run: read(stage, part) and
// compute(part), for the PARTS parts of a stage. A stage's place is loaded again once
// the later half has read it, one phase after the earlier half. (Sent out
// beside the matrix instructions instead of the reads, the loads cost 7%.)
template <class Shape, int PARTS, class Issue, class Read, class Compute>
__device__ inline void run_alternating(int32_t count, const short *lds, int wave, Issue issue,
                                       Read read, Compute compute) {
    static_assert(Shape::kWaves == 8, "two waves on each SIMD");
    constexpr int kAny = Shape::STAGES * Shape::kLoads;
    constexpr int kOpen = (Shape::STAGES - 2) * Shape::kLoads;
#pragma unroll
    for (int s = 0; s < Shape::STAGES - 1; ++s) issue(lds + s * Shape::kStage);
    const short *reads = lds, *writes = lds + (Shape::STAGES - 1) * Shape::kStage;
    const short *end = lds + Shape::kLds;
    auto next = [&](const short *p) {
        p += Shape::kStage;
        return p == end ? lds : p;
    };
    phase<kOpen>();
    if (wave >= 4)
        phase<kOpen>();
    for (int32_t it = 0; it < count; ++it) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            read(reads, part);
            if (part == 0)
                issue(writes);
            // the next stage has landed when this one's last part has been read
            if (part + 1 == PARTS)
                phase<kOpen>();
            else
                phase<kAny>();
            __builtin_amdgcn_s_setprio(1);
            compute(part);
            __builtin_amdgcn_s_setprio(0);
            phase<kAny>();
        }
        reads = next(reads);
        writes = next(writes);
    }
    if (wave < 4)
        phase<kAny>();
    meet<0>();
}

// acc[i][j][r] += D at row 16 i + lane % 16 and column 16 j + 4 (lane / 16) + r of
// the wave's part, over `depth` values of k.
//
// With two parts, `low_a` and `low_b` bytes apart, it sums the products high low, low
// high and high high. A matrix instruction rounds each of its products to the
// accumulator's last place, which costs a chain over k = 1024 about 1e-6; so 32 values
// of k are summed from 0, small products first, and added to the accumulator in one
// rounding. Sums of at most kFewTerms, whose few roundings do not average out, take the
// product low low as well (not in the alternating form): orthogonalized 12 x 10 matrices
// end 5.5e-7 off in the median, 6.9e-7 without, in plain fp32 7.0e-7; 161 x 59 ones 1.0e-6,
// 1.4e-6 and 1.4e-6.
constexpr int32_t kFewTerms = 64;
template <class Math, class Shape, bool COLS_A, bool COLS_B>
__device__ inline void tile_product(float4v (&acc)[Shape::MI][Shape::NI], const short *lds,
                                    const Operand &a, const Operand &b, int64_t depth,
                                    int64_t low_a = 0, int64_t low_b = 0) {
    constexpr int D = Shape::DEPTH, kA = Shape::kA, kB = Shape::kB;
    constexpr bool kSplit = Shape::PARTS == 2;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Shape::WN, wn = wave % Shape::WN;
    StageLoader<Shape::BM, D, Shape::kWaves, COLS_A> la;
    StageLoader<Shape::BN, D, Shape::kWaves, COLS_B> lb;
    la.init(a, wave, lane);
    lb.init(b, wave, lane);
    const int64_t step_a = COLS_A ? a.ld * D : D * 2;
    const int64_t step_b = COLS_B ? b.ld * D : D * 2;
    int32_t left = int32_t(depth);
    const char *pa = a.base, *pb = b.base;
    auto issue = [&](const short *s) {
        la.issue(pa, left, s, wave);
        if (kSplit)
            la.issue(pa + low_a, left, s + kA, wave);
        lb.issue(pb, left, s + Shape::PARTS * kA, wave);
        if (kSplit)
            lb.issue(pb + low_b, left, s + 2 * kA + kB, wave);
        left -= D;
        if (left > 0) {
            pa += step_a;
            pb += step_b;
        }
    };
    auto read_a = [&](const short *s, int i, int step) {
        return read_fragment<Shape::BM, D, COLS_A>(s, (wm * Shape::MI + i) * 16, step, lane);
    };
    auto read_b = [&](const short *s, int j, int step) {
        return read_fragment<Shape::BN, D, COLS_B>(s + Shape::PARTS * kA,
                                                   (wn * Shape::NI + j) * 16, step, lane);
    };
    const int32_t count = int32_t((depth + D - 1) / D);
    if constexpr (Shape::kAlternating) {
        static_assert(D == 32, "a stage is one step");
        // two parts keep a split product's fragments within the registers
        constexpr int kParts = Shape::PARTS, kRows = Shape::MI / kParts;
        short8v fa[Shape::PARTS][kRows], fb[Shape::PARTS][Shape::NI];
        run_alternating<Shape, kParts>(
            count, lds, wave, issue,
            [&](const short *s, int part) {
#pragma unroll
                for (int p = 0; p < Shape::PARTS; ++p) {
                    if (part == 0) {
#pragma unroll
                        for (int j = 0; j < Shape::NI; ++j) fb[p][j] = read_b(s + p * kB, j, 0);
                    }
#pragma unroll
                    for (int i = 0; i < kRows; ++i)
                        fa[p][i] = read_a(s + p * kA, part * kRows + i, 0);
                }
            },
            [&](int part) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    float4v(&to)[Shape::NI] = acc[part * kRows + i];
                    if constexpr (!kSplit) {
#pragma unroll
                        for (int j = 0; j < Shape::NI; ++j)
                            to[j] = Math::mma(fb[0][j], fa[0][i], to[j]);
                    } else {
                        float4v sum[Shape::NI];
#pragma unroll
                        for (int j = 0; j < Shape::NI; ++j)
                            sum[j] = Math::mma(fb[0][j], fa[1][i], float4v{});
#pragma unroll
                        for (int j = 0; j < Shape::NI; ++j)
                            sum[j] = Math::mma(fb[1][j], fa[0][i], sum[j]);
#pragma unroll
                        for (int j = 0; j < Shape::NI; ++j)
                            sum[j] = Math::mma(fb[0][j], fa[0][i], sum[j]);
#pragma unroll
                        for (int j = 0; j < Shape::NI; ++j)
#pragma unroll
                            for (int r = 0; r < 4; ++r) to[j][r] += sum[j][r];
                    }
                }
            });
        return;
    }
    auto compute = [&](const short *s, auto few) {
#pragma unroll
        for (int step = 0; step < D / 32; ++step) {
            short8v fb[Shape::PARTS][Shape::NI];
#pragma unroll
            for (int p = 0; p < Shape::PARTS; ++p)
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j) fb[p][j] = read_b(s + p * kB, j, step);
#pragma unroll
            for (int i = 0; i < Shape::MI; ++i) {
                const short8v hi = read_a(s, i, step);
                if (!kSplit) {
#pragma unroll
                    for (int j = 0; j < Shape::NI; ++j)
                        acc[i][j] = Math::mma(fb[0][j], hi, acc[i][j]);
                    continue;
                }
                const short8v lo = read_a(s + kA, i, step);
                float4v part[Shape::NI] = {};
                if (decltype(few)::value) {
#pragma unroll
                    for (int j = 0; j < Shape::NI; ++j)
                        part[j] = Math::mma(fb[kSplit][j], lo, part[j]);
                }
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j) part[j] = Math::mma(fb[0][j], lo, part[j]);
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j)
                    part[j] = Math::mma(fb[kSplit][j], hi, part[j]);
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j) part[j] = Math::mma(fb[0][j], hi, part[j]);
#pragma unroll
                for (int j = 0; j < Shape::NI; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] += part[j][r];
            }
        }
    };
    if (kSplit && depth <= kFewTerms)
        run_stages<Shape>(count, lds, issue,
                          [&](const short *s) { compute(s, std::true_type{}); });
    else
        run_stages<Shape>(count, lds, issue,
                          [&](const short *s) { compute(s, std::false_type{}); });
}

// The lane's first value of acc in the tile.
template <class Shape>
struct Place {
    int row, col;
    __device__ Place() {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        row = wave / Shape::WN * (Shape::BM / Shape::WM) + (lane & 15);
        col = wave % Shape::WN * (Shape::BN / Shape::WN) + 4 * (lane >> 4);
    }
};

// A tile of 16-bit values leaves through LDS, so that rows are written 16 bytes a lane:
// put() writes the lane's four of row m, columns n .. n + 3 (MIRROR: of column m, rows
// n .. n + 3 of the transposed tile), flush() stores the tile's rows. 16-byte pieces
// are swapped within a row, by slot(), to spread the banks. All of the workgroup takes
// part; LDS must hold ROWS x COLS elements.
template <int ROWS, int COLS, int THREADS>
struct TileStore {
    static constexpr int kPieces = COLS / 8;
    static constexpr int kMask = kPieces < 8 ? kPieces - 1 : 7;
    short *lds;
    __device__ explicit TileStore(short *p) : lds(p) {}
    static __device__ int at(int row, int col, int slot) {
        return row * COLS + (((col >> 3) ^ (slot & kMask)) << 3) + (col & 7);
    }
    __device__ void put(int m, int n, ushort4 v) const { *(ushort4 *)(lds + at(m, n, m)) = v; }
    __device__ void put_mirror(int m, int n, ushort4 v) const {
        lds[at(n, m, n >> 2)] = short(v.x);
        lds[at(n + 1, m, n >> 2)] = short(v.y);
        lds[at(n + 2, m, n >> 2)] = short(v.z);
        lds[at(n + 3, m, n >> 2)] = short(v.w);
    }
    // Rows and columns below the limits, from `to` with `ld` elements a row; the column
    // limit is a multiple of 8.
    template <bool MIRROR>
    __device__ void flush(uint16_t *to, int64_t ld, int rows, int cols) const {
        __syncthreads();
#pragma unroll 4
        for (int p = threadIdx.x; p < ROWS * kPieces; p += THREADS) {
            const int row = p / kPieces, col = p % kPieces * 8;
            if (row < rows && col < cols)
                store_global(to + row * ld + col,
                             *(const uint4 *)(lds + at(row, col, MIRROR ? row >> 2 : row)));
        }
        __syncthreads();
    }
};

}  // namespace lamb_mi355x
