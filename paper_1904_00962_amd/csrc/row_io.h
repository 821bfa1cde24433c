// Eight elements of a row at a time, float32 or bfloat16, in the registers of one lane:
// what the kernels that stream rows or lists of tensors share. Not installed.
//
// A lane's eight elements are loaded and stored in pieces of 16 bytes that are aligned to
// an element only: the hardware takes them at any address, so rows of odd widths and
// tensors that begin anywhere need no other path.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace lamb_mi355x {

__device__ inline float bf16_low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ inline float bf16_high(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

__device__ inline uint32_t bf16_pair(float low, float high) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 both = {__bf16(low), __bf16(high)};
    return __builtin_bit_cast(uint32_t, both);
}

// Device memory: accesses through pointers that a kernel has read from memory need not look
// which kind of memory it is.
template <class T>
using Global = __attribute__((address_space(1))) T;

// 16 bytes that begin at any element.
typedef uint32_t Bytes16 __attribute__((ext_vector_type(4), aligned(2)));

template <bool STREAM>
__device__ inline Bytes16 load_16(const Global<void> *p) {
    const Global<Bytes16> *from = (const Global<Bytes16> *)p;
    return STREAM ? __builtin_nontemporal_load(from) : *from;
}

template <bool STREAM>
__device__ inline void store_16(Global<void> *p, Bytes16 v) {
    Global<Bytes16> *to = (Global<Bytes16> *)p;
    if (STREAM)
        __builtin_nontemporal_store(v, to);
    else
        *to = v;
}

// Eight elements as they lie in memory.
template <bool BF16>
struct Eight {
    uint32_t u[BF16 ? 4 : 8];

    __device__ inline void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (BF16) {
                v[2 * i] = bf16_low(u[i]);
                v[2 * i + 1] = bf16_high(u[i]);
            } else {
                v[2 * i] = __uint_as_float(u[BF16 ? 0 : 2 * i]);
                v[2 * i + 1] = __uint_as_float(u[BF16 ? 0 : 2 * i + 1]);
            }
        }
    }
    __device__ inline void set(const float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (BF16) {
                u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
            } else {
                u[BF16 ? 0 : 2 * i] = __float_as_uint(v[2 * i]);
                u[BF16 ? 0 : 2 * i + 1] = __float_as_uint(v[2 * i + 1]);
            }
        }
    }
};

// Moves the elements `by` places (0 to 7) towards the first; zeros follow.
template <bool BF16>
__device__ inline void move_down(Eight<BF16> &e, int by) {
    constexpr int kWords = BF16 ? 4 : 8;
    if (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t above = i < 3 ? e.u[i < 3 ? i + 1 : 3] : 0u;
            e.u[i] = by & 1 ? above << 16 | e.u[i] >> 16 : e.u[i];
        }
        by >>= 1;
    }
#pragma unroll
    for (int step = 1; step < kWords; step *= 2)
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const uint32_t above = i + step < kWords ? e.u[(i + step) % kWords] : 0u;
            e.u[i] = by & step ? above : e.u[i];
        }
}

// Elements at .. at + n - 1 of `base` (n below 1: none); what is past them is 0, once
// settled. Where the eight that end with the last of them may be read (`back`), a row's last
// few take the same one load, of those eight, and settle() moves them to their places: later,
// so that no load waits for another's end. TAIL false: n is at least 8, or below 1; rows of
// whole eights go faster where nothing else is compiled in (32768 rows of 1600: the 8-bit
// norm 62 us in place of 69, the gradients 126 in place of 157).
template <bool BF16, bool TAIL, bool STREAM = false>
__device__ inline Eight<BF16> load_eight(const void *base, int64_t at, int n, bool back = false) {
    using T = typename std::conditional<BF16, uint16_t, uint32_t>::type;
    Eight<BF16> e = {};
    const Global<T> *p = (const Global<T> *)base + at;
    if (n >= 8 || (TAIL && back && n > 0)) {
        if (TAIL)
            p -= n < 8 ? 8 - n : 0;
        const Bytes16 a = load_16<STREAM>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) e.u[i] = a[i];
        if (!BF16) {
            const Bytes16 b = load_16<STREAM>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) e.u[BF16 ? 0 : i + 4] = b[i];
        }
    } else if (TAIL && n > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n)
                e.u[BF16 ? i / 2 : i] |= uint32_t(p[i]) << (BF16 ? i % 2 * 16 : 0);
    }
    return e;
}

template <bool TAIL, bool BF16>
__device__ inline void settle(Eight<BF16> &e, int n, bool back) {
    if (TAIL && back && n > 0 && n < 8) {
        asm volatile("");  // stays a branch: as selects the moves would cost every lane
        move_down(e, 8 - n);
    }
}

template <bool BF16, bool TAIL, bool STREAM = false>
__device__ inline void store_eight(void *base, int64_t at, int n, const Eight<BF16> &e) {
    if (BF16) {
        Global<uint16_t> *p = (Global<uint16_t> *)base + at;
        if (n >= 8) {
            store_16<STREAM>(p, Bytes16{e.u[0], e.u[1], e.u[2], e.u[3]});
        } else if (TAIL && n > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n)
                    p[i] = uint16_t(e.u[i / 2] >> (i % 2 * 16));
        }
    } else {
        Global<uint32_t> *p = (Global<uint32_t> *)base + at;
        if (n >= 8) {
            store_16<STREAM>(p, Bytes16{e.u[0], e.u[1], e.u[2], e.u[3]});
            store_16<STREAM>(p + 4, Bytes16{e.u[BF16 ? 0 : 4], e.u[BF16 ? 0 : 5],
                                             e.u[BF16 ? 0 : 6], e.u[BF16 ? 0 : 7]});
        } else if (TAIL && n > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n)
                    p[i] = e.u[BF16 ? 0 : i];
        }
    }
}

// The same with a type that is known at run time only, for what is not on a kernel's
// longest path.
template <bool BF16, bool TAIL>
__device__ inline void load_values_of(const void *base, int64_t at, int n, bool back,
                                      float (&v)[8]) {
    Eight<BF16> e = load_eight<BF16, TAIL>(base, at, n, back);
    settle<TAIL>(e, n, back);
    e.get(v);
}

template <bool TAIL>
__device__ inline void load_values(bool bf16, const void *base, int64_t at, int n, bool back,
                                   float (&v)[8]) {
    if (bf16)
        load_values_of<true, TAIL>(base, at, n, back, v);
    else
        load_values_of<false, TAIL>(base, at, n, back, v);
}

template <bool TAIL, bool STREAM = false>
__device__ inline void store_values(bool bf16, void *base, int64_t at, int n,
                                    const float (&v)[8]) {
    if (bf16) {
        Eight<true> e;
        e.set(v);
        store_eight<true, TAIL, STREAM>(base, at, n, e);
    } else {
        Eight<false> e;
        e.set(v);
        store_eight<false, TAIL, STREAM>(base, at, n, e);
    }
}

}  // namespace lamb_mi355x
