// Eight elements of a row at a time, float32 or bfloat16, in the registers of one lane:
// what the kernels that stream rows or lists of tensors share. Not installed.
//
// A lane's eight elements are loaded and stored in pieces of 16 bytes that are aligned to
// an element only: the hardware takes them at any address, so rows of odd widths and
// tensors that begin anywhere need no other path.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

// Elements at .. at + n - 1 of `base` (n below 1: none); what is past them is 0.
template <bool BF16, bool STREAM = false>
__device__ inline Eight<BF16> load_eight(const void *base, int64_t at, int n) {
    Eight<BF16> e;
    if (BF16) {
        const Global<uint16_t> *p = (const Global<uint16_t> *)base + at;
        if (n >= 8) {
            const Bytes16 w = load_16<STREAM>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) e.u[i] = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                e.u[i] = (2 * i < n ? uint32_t(p[2 * i]) : 0u) |
                         (2 * i + 1 < n ? uint32_t(p[2 * i + 1]) << 16 : 0u);
        }
    } else {
        const Global<uint32_t> *p = (const Global<uint32_t> *)base + at;
        if (n >= 8) {
            const Bytes16 a = load_16<STREAM>(p), b = load_16<STREAM>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e.u[i] = a[i];
                e.u[BF16 ? 0 : i + 4] = b[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e.u[BF16 ? 0 : i] = i < n ? p[i] : 0u;
        }
    }
    return e;
}

template <bool BF16, bool STREAM = false>
__device__ inline void store_eight(void *base, int64_t at, int n, const Eight<BF16> &e) {
    if (BF16) {
        Global<uint16_t> *p = (Global<uint16_t> *)base + at;
        if (n >= 8) {
            store_16<STREAM>(p, Bytes16{e.u[0], e.u[1], e.u[2], e.u[3]});
        } else {
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
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n)
                    p[i] = e.u[BF16 ? 0 : i];
        }
    }
}

// The same with a type that is known at run time only, for what is not on a kernel's
// longest path.
__device__ inline void load_values(bool bf16, const void *base, int64_t at, int n,
                                   float (&v)[8]) {
    if (bf16)
        load_eight<true>(base, at, n).get(v);
    else
        load_eight<false>(base, at, n).get(v);
}

template <bool STREAM = false>
__device__ inline void store_values(bool bf16, void *base, int64_t at, int n,
                                    const float (&v)[8]) {
    if (bf16) {
        Eight<true> e;
        e.set(v);
        store_eight<true, STREAM>(base, at, n, e);
    } else {
        Eight<false> e;
        e.set(v);
        store_eight<false, STREAM>(base, at, n, e);
    }
}

}  // namespace lamb_mi355x
