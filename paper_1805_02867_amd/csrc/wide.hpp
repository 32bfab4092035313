// Binary64 building blocks of the kernels whose choices must not depend on
// rounding: sampling (a vocabulary of 10^5 has as many borders that a random
// number can fall on) and routing (a bias brings scores close together).  CDNA
// vector units take a binary64 fma at the rate of a binary32 one, so these cost
// registers, not time.
#pragma once

#include "md.hpp"

namespace osm {

constexpr double kLog2eD = 1.4426950408889634074;

// 2^t for t <= 1023, to 3e-16: n + f = t with |f| <= 1/2, 2^f = 1 + f g(f) with g
// the polynomial through (2^f - 1) / f at the eleven Chebyshev nodes of
// [-1/2, 1/2] (truncation 2e-17), so that 2^0 is 1 exactly.  Below 2^-1074, at
// -inf and at NaN: 0.
__device__ __forceinline__ double exp2_wide(double t) {
    t = __builtin_fmax(t, -1100.0);
    const double n = __builtin_rint(t);
    const double f = t - n;
    double g = 0x1.e9d3fe3952179p-32;
    g = __builtin_fma(g, f, 0x1.e6063f7217bc6p-28);
    g = __builtin_fma(g, f, 0x1.b524fae627834p-24);
    g = __builtin_fma(g, f, 0x1.62bfd47773353p-20);
    g = __builtin_fma(g, f, 0x1.ffcbfc670dcd4p-17);
    g = __builtin_fma(g, f, 0x1.430913096fd9fp-13);
    g = __builtin_fma(g, f, 0x1.5d87fe78a5276p-10);
    g = __builtin_fma(g, f, 0x1.3b2ab6fba1ddap-7);
    g = __builtin_fma(g, f, 0x1.c6b08d704a0c2p-5);
    g = __builtin_fma(g, f, 0x1.ebfbdff82c598p-3);
    g = __builtin_fma(g, f, 0x1.62e42fefa39efp-1);
    return __builtin_ldexp(__builtin_fma(g, f, 1.0), (int)n);
}

// Butterfly operands (md.hpp) of a 64-bit value.
template <int STEP>
__device__ __forceinline__ void bfly_operands64(uint64_t v, uint64_t& a, uint64_t& b) {
    uint32_t al, bl, ah, bh;
    bfly_operands<STEP>((uint32_t)v, al, bl);
    bfly_operands<STEP>((uint32_t)(v >> 32), ah, bh);
    a = (uint64_t)ah << 32 | al;
    b = (uint64_t)bh << 32 | bl;
}

// Sum over aligned groups of G lanes; every lane gets the same bits.
template <int G, int STEP = 0>
__device__ __forceinline__ double group_sum(double v) {
    if constexpr ((1 << STEP) < G) {
        uint64_t a, b;
        bfly_operands64<STEP>(__builtin_bit_cast(uint64_t, v), a, b);
        return group_sum<G, STEP + 1>(__builtin_bit_cast(double, a) +
                                      __builtin_bit_cast(double, b));
    } else {
        return v;
    }
}

// Largest value over aligned groups of G lanes, every lane gets it.
template <int G, int STEP = 0>
__device__ __forceinline__ uint64_t group_max(uint64_t v) {
    if constexpr ((1 << STEP) < G) {
        uint64_t a, b;
        bfly_operands64<STEP>(v, a, b);
        return group_max<G, STEP + 1>(a > b ? a : b);
    } else {
        return v;
    }
}

template <int G, int STEP = 0>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    if constexpr ((1 << STEP) < G) {
        uint32_t a, b;
        bfly_operands<STEP>(v, a, b);
        return group_max<G, STEP + 1>(a > b ? a : b);
    } else {
        return v;
    }
}

// Inclusive prefix sum over the wavefront's lanes.
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const V o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Order of values as unsigned integers; -0.0 ranks as +0.0.
__device__ __forceinline__ uint32_t order_key(float x) {
    uint32_t u = __float_as_uint(x);
    u = u == 0x80000000u ? 0u : u;
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float order_value(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

__device__ __forceinline__ uint64_t order_key(double x) {
    uint64_t u = __builtin_bit_cast(uint64_t, x);
    u = u == 0x8000000000000000ull ? 0ull : u;
    return u ^ ((uint64_t)((int64_t)u >> 63) | 0x8000000000000000ull);
}

__device__ __forceinline__ double order_value64(uint64_t k) {
    return __builtin_bit_cast(double, (k & 0x8000000000000000ull) ? (k & 0x7FFFFFFFFFFFFFFFull)
                                                                  : ~k);
}

}  // namespace osm
