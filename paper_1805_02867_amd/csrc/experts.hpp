// Rows of router logits in registers: a row by a team of 8 to 64 lanes.
#pragma once

#include "wide.hpp"

namespace osm {

// The row team of a lane: LANES lanes, `lane` within it.  Lane l's j-th expert is
// (j / VEC * LANES + l) * VEC + j % VEC: VEC neighbours are loaded together.
template <int LANES, int VEC>
__device__ __forceinline__ int expert(int lane, int j) {
    return (j / VEC * LANES + lane) * VEC + j % VEC;
}

template <typename T, int LANES, int R, int VEC>
__device__ __forceinline__ void load_experts(const T* xr, int E, bool live, int lane,
                                             float (&x)[R]) {
    if constexpr (VEC == 1) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int e = j * LANES + lane;
            x[j] = live && e < E ? load1(xr + e) : -__builtin_inff();
        }
    } else {
#pragma unroll
        for (int j = 0; j < R; j += 4) {
            const int e = expert<LANES, VEC>(lane, j);
#pragma unroll
            for (int v = 0; v < 4; ++v) x[j + v] = -__builtin_inff();
            if (!live || e >= E) continue;
            if constexpr (sizeof(T) == 4) {
                const f32x4 q = *reinterpret_cast<const f32x4*>(xr + e);
#pragma unroll
                for (int v = 0; v < 4; ++v) x[j + v] = q[v];
            } else {
                const uint2 q = *reinterpret_cast<const uint2*>(xr + e);
                x[j] = bf16_lo(q.x);
                x[j + 1] = bf16_hi(q.x);
                x[j + 2] = bf16_lo(q.y);
                x[j + 3] = bf16_hi(q.y);
            }
        }
    }
}

template <typename T, int LANES, int R, int VEC>
__device__ __forceinline__ void store_experts(T* dr, int E, int lane, const float (&d)[R]) {
    if constexpr (VEC == 1) {
#pragma unroll
        for (int j = 0; j < R; ++j)
            if (j * LANES + lane < E) store1(dr + j * LANES + lane, d[j]);
    } else {
#pragma unroll
        for (int j = 0; j < R; j += 4) {
            const int e = expert<LANES, VEC>(lane, j);
            if (e >= E) continue;
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<f32x4*>(dr + e) = f32x4{d[j], d[j + 1], d[j + 2], d[j + 3]};
            else
                *reinterpret_cast<uint2*>(dr + e) =
                    uint2{pack_bf16x2(d[j], d[j + 1]), pack_bf16x2(d[j + 2], d[j + 3])};
        }
    }
}

template <int LANES>
__device__ __forceinline__ float team_maximum(float v) {  // (NaN where there is one)
    float a, b;
#define OSM_STEP(S)                                              \
    if constexpr (LANES > (1 << S)) {                            \
        bfly_operands<S>(v, a, b);                               \
        v = __builtin_elementwise_maximum(a, b);                 \
    }
    OSM_STEP(0) OSM_STEP(1) OSM_STEP(2) OSM_STEP(3) OSM_STEP(4) OSM_STEP(5)
#undef OSM_STEP
    return v;
}

}  // namespace osm
