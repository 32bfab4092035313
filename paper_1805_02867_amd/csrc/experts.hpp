// Rows of router logits in registers: a row by a team of 8 to 64 lanes.
#pragma once

#include <type_traits>

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

// A row's experts as they come from memory: every lane loads, from a place inside the row where
// it has no expert, so that nothing waits; `widen` makes numbers of them, -inf where there is no
// expert.
template <typename T, int LANES, int R, int VEC>
struct RawExperts {
    using V4 = std::conditional_t<sizeof(T) == 4, f32x4, uint2>;
    using V1 = std::conditional_t<sizeof(T) == 4, float, uint16_t>;
    static constexpr int N = VEC == 4 ? R / 4 : R;
    using V = std::conditional_t<VEC == 4, V4, V1>;
    V q[N];

    // at: the row's place behind `base`, in bytes.
    __device__ __forceinline__ void load(const char* base, uint32_t at, int E, int lane) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = expert<LANES, VEC>(lane, i * VEC);
            q[i] = *reinterpret_cast<const V*>(base + (at + (uint32_t)(e < E ? e : 0) *
                                                                (uint32_t)sizeof(T)));
        }
    }
    // FULL: there is an expert in every place.
    template <bool FULL>
    __device__ __forceinline__ void widen(float (&x)[R], int E, int lane) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool in = FULL || expert<LANES, VEC>(lane, i * VEC) < E;
            float v[VEC];
            if constexpr (VEC == 4 && sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = q[i][k];
            } else if constexpr (VEC == 4) {
                v[0] = bf16_lo(q[i].x), v[1] = bf16_hi(q[i].x);
                v[2] = bf16_lo(q[i].y), v[3] = bf16_hi(q[i].y);
            } else if constexpr (sizeof(T) == 4) {
                v[0] = q[i];
            } else {
                v[0] = __uint_as_float((uint32_t)q[i] << 16);
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[i * VEC + k] = in ? v[k] : -__builtin_inff();
        }
    }
};

// Sum over the wavefront's teams of what the lanes with the same place in them hold.
template <int LANES>
__device__ __forceinline__ float sum_of_teams(float v) {
    float a, b;
    if constexpr (LANES <= 8)  // a rotation by 8 within 16 lanes
        v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
            0, (int)__float_as_uint(v), 0x128, 0xF, 0xF, false));
    if constexpr (LANES <= 16) {
        bfly_operands<4>(v, a, b);
        v = a + b;
    }
    if constexpr (LANES <= 32) {
        bfly_operands<5>(v, a, b);
        v = a + b;
    }
    return v;
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
