// Binary64 building blocks of the kernels whose choices must not depend on
// rounding: sampling (a vocabulary of 10^5 has as many borders that a random
// number can fall on) and routing (a bias brings scores close together).  CDNA
// vector units take a binary64 fma at the rate of a binary32 one; what these cost is
// registers, and the instructions of a polynomial where binary32 has one for 2^t.
#pragma once

#include "md.hpp"

namespace osm {

constexpr double kLog2eD = 1.4426950408889634074;

// A constant kept in scalar registers.  As a literal the compiler moves it into vector
// registers for every use, as the sum that an accumulating fma overwrites: two moves an
// fma, most of the cost of a polynomial.
__device__ __forceinline__ double scalar(double c) {
    asm("" : "+s"(c));
    return c;
}

// 2^t for -2^30 < t <= 1023, to 7e-16: n + f = t with |f| <= 1/2, 2^f = 1 + f g(f) with g
// the polynomial through (2^f - 1) / f at the ten Chebyshev nodes of [-1/2, 1/2]
// (truncation 6e-16), so that 2^0 is 1 exactly.  Below 2^-1074: 0.  Made once and
// handed to a loop, so that its constants stay where they are.
struct Exp2 {
    double k[10];
    __device__ __forceinline__ static Exp2 make() {
        return Exp2{{scalar(0x1.e5e9f548e5725p-28),
                     scalar(0x1.b6571de2f2351p-24),
                     scalar(0x1.62bfe46117445p-20),
                     scalar(0x1.ffcb76789860fp-17),
                     scalar(0x1.4309130378460p-13),
                     scalar(0x1.5d87fe908f88ap-10),
                     scalar(0x1.3b2ab6fba385fp-7),
                     scalar(0x1.c6b08d7044119p-5),
                     scalar(0x1.ebfbdff82c590p-3),
                     scalar(0x1.62e42fefa39f7p-1)}};
    }
    __device__ __forceinline__ double operator()(double t) const {
        const double n = __builtin_rint(t);
        const double f = t - n;
        double g = k[0];
#pragma unroll
        for (int i = 1; i < 10; ++i) g = __builtin_fma(g, f, k[i]);
        return __builtin_ldexp(__builtin_fma(g, f, 1.0), (int)n);
    }
};

__device__ __forceinline__ double exp2_bounded(double t) { return Exp2::make()(t); }

// The same for any t <= 1023; 0 at -inf and at NaN.
__device__ __forceinline__ double exp2_wide(double t) {
    return exp2_bounded(__builtin_fmax(t, -1100.0));
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

// Inclusive prefix sum over the wavefront's lanes, in cross-lane VALU moves: within rows
// of 16 lanes by shifts of 1, 2, 4 and 8, then the last lane of row 0 (2) is added
// to row 1 (3), and that of the lower half to the upper one.  Lanes a move does not
// reach add 0.  All lanes must be active.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_or_zero(uint64_t v) {
    return (uint64_t)dpp_or_zero<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 |
           dpp_or_zero<CTRL, ROWS>((uint32_t)v);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_or_zero(double v) {
    return __builtin_bit_cast(double, dpp_or_zero<CTRL, ROWS>(__builtin_bit_cast(uint64_t, v)));
}
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
    v += dpp_or_zero<0x111, 0xF>(v);  // row_shr:1
    v += dpp_or_zero<0x112, 0xF>(v);
    v += dpp_or_zero<0x114, 0xF>(v);
    v += dpp_or_zero<0x118, 0xF>(v);
    v += dpp_or_zero<0x142, 0xA>(v);  // row_bcast:15 into rows 1 and 3
    v += dpp_or_zero<0x143, 0xC>(v);  // row_bcast:31 into rows 2 and 3
    return v;
}
// The value of the lane before (0 in lane 0), and of one lane.
template <typename V>
__device__ __forceinline__ V lane_before(V v) {
    return dpp_or_zero<0x138, 0xF>(v);  // wave_shr:1
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) {
    return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    return (uint64_t)lane_value((uint32_t)(v >> 32), lane) << 32 | lane_value((uint32_t)v, lane);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
    return __builtin_bit_cast(double, lane_value(__builtin_bit_cast(uint64_t, v), lane));
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(lane_value(__float_as_uint(v), lane));
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
