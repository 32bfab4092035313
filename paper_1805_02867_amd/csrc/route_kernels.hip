// Routing tokens to experts, and the gradient of the weights.
//
// Forward, a row of E logits x: scores s = softmax(x) or 1 / (1 + e^-x); experts
// are ranked by c = s + bias, or by x itself without a bias (both scores
// increase with x); with groups, each group of E / G experts is ranked by the
// sum of its group_top best, and only the best top_groups are searched; the K
// largest c, ties to the lower index, give the experts, and their s the weights
// (renormalised to sum 1 if asked, times scale).  Renormalised weights are
// taken from the chosen logits alone, relative to the largest, so they do not
// underflow together.
//
// Scores are binary64: a bias brings experts close together, and a choice must
// not depend on the order of a sum.
//
// Backward, with g the gradient of the K weights and p = weights / scale:
//   softmax, renormalised:  dx_i = scale p_i (g_i - sum_j g_j p_j) at the chosen
//   softmax:                dx_e = scale s_e (g_e - sum_j g_j s_j), everywhere
//   sigmoid, renormalised:  dx_i = scale p_i (g_i - sum_j g_j p_j) (1 - s_i)
//   sigmoid:                dx_i = scale g_i s_i (1 - s_i)
// and 0 elsewhere.  The choice itself has no gradient, and neither has the bias.
#include "wide.hpp"
#include "kernels.h"

namespace osm {

constexpr int RT_BLOCK = 256;
constexpr int RT_WAVES = RT_BLOCK / 64;
constexpr int RT_EMAX = 1024;
constexpr int RT_GMAX = 64;

__device__ __forceinline__ double sigmoid_wide(double x) {
    const double e = exp2_wide(-__builtin_fabs(x) * kLog2eD);
    return (x >= 0.0 ? 1.0 : e) / (1.0 + e);
}

// Experts that cannot be chosen rank here, below every score (even -1e308).
constexpr uint64_t kNoRank = 0;

// A wavefront per row; lane l holds experts l, l + 64, ...
template <typename T, int R>
__global__ __launch_bounds__(RT_BLOCK) void route_rows(const RouteRows a) {
    __shared__ uint64_t ranks[RT_WAVES][RT_EMAX];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int E = a.E, K = a.K;
    const double inf = __builtin_inf();
    uint64_t* const rk = ranks[wv];
    for (int64_t row = (int64_t)blockIdx.x * RT_WAVES + wv; row < a.N;
         row += (int64_t)gridDim.x * RT_WAVES) {
        const T* xr = static_cast<const T*>(a.x) + row * E;
        float x[R];
        float mx = -__builtin_inff();
        bool bad = false;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int e = j * 64 + lane;
            x[j] = e < E ? load1(xr + e) : -__builtin_inff();
            bad |= !(x[j] < __builtin_inff());
            mx = fmaxf(mx, x[j]);
        }
        mx = group_max<64>(mx);
        bad = __any(bad);
        if (bad || mx == -__builtin_inff()) {
            if (lane < K) {
                a.idx[row * K + lane] = -1;
                a.vals[row * K + lane] = bad ? __builtin_nanf("") : 0.0f;
            }
            continue;
        }
        // scores
        double s[R], sum = 0.0;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            s[j] = a.sigmoid ? sigmoid_wide((double)x[j])
                             : exp2_wide(((double)x[j] - (double)mx) * kLog2eD);
            sum += s[j];
        }
        if (!a.sigmoid) {
            sum = group_sum<64>(sum);
#pragma unroll
            for (int j = 0; j < R; ++j) s[j] /= sum;
        }
        // ranks
        uint64_t r[R];
        double b[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int e = j * 64 + lane;
            b[j] = a.bias && e < E ? (double)a.bias[e] : 0.0;
            const bool may = x[j] > -__builtin_inff() && b[j] > -inf;  // (NaN bias: no)
            r[j] = !may ? kNoRank : order_key(a.bias ? s[j] + b[j] : (double)x[j]);
        }
        if (a.groups > 1) {
            // the score of group `lane`, from its best one or two experts
            const int gs = E / a.groups;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int e = j * 64 + lane;
                if (e < E) rk[e] = r[j] == kNoRank ? kNoRank : order_key(s[j] + b[j]);
            }
            wave_sync();
            uint64_t best = 0, second = 0;
            if (lane < a.groups) {
                for (int i = 0; i < gs; ++i) {
                    const uint64_t k = rk[lane * gs + i];
                    second = k > best ? best : k > second ? k : second;
                    best = k > best ? k : best;
                }
            }
            uint64_t g = best;
            if (a.group_top == 2 && second != kNoRank)
                g = order_key(order_value64(best) + order_value64(second));
            int ahead = 0;
            for (int o = 0; o < a.groups; ++o) {
                const uint64_t k = __shfl(g, o);
                ahead += k > g || (k == g && o < lane);
            }
            const uint64_t keep = __ballot(lane < a.groups && ahead < a.top_groups);
            wave_sync();
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int e = j * 64 + lane;
                if (e >= E || !(keep >> (e / gs) & 1)) r[j] = kNoRank;
            }
        }
        // K times the largest rank, ties to the lower index
        int mine = -1;
        float mx_in = 0.0f;
        for (int i = 0; i < K; ++i) {
            uint64_t best = 0;
            int at = 0;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                at = r[j] > best ? j : at;
                best = r[j] > best ? r[j] : best;
            }
            const uint64_t top = group_max<64>(best);
            if (top == kNoRank) break;
            // the lowest index of that rank
            uint32_t e = best == top ? (uint32_t)(at * 64 + lane) : ~0u;
            e = ~group_max<64>(~e);
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (e == (uint32_t)(j * 64 + lane)) r[j] = kNoRank;
            mine = lane == i ? (int)e : mine;
        }
        // weights: lane i has the i-th expert
        double w = 0.0;
        if (mine >= 0) {
            mx_in = load1(xr + mine);
            w = a.sigmoid ? sigmoid_wide((double)mx_in)
                          : exp2_wide(((double)mx_in - (double)mx) * kLog2eD) / sum;
        }
        if (a.renorm) {
            // relative to the largest chosen one: e^x, or e^min(x, 0) / (1 + e^-|x|)
            const double z = mine < 0   ? -inf
                             : a.sigmoid ? __builtin_fmin((double)mx_in, 0.0)
                                         : (double)mx_in;
            const double zm = (double)group_max<64>((float)z);
            w = exp2_wide((z - zm) * kLog2eD);
            if (a.sigmoid) w /= 1.0 + exp2_wide(-__builtin_fabs((double)mx_in) * kLog2eD);
            w = mine < 0 ? 0.0 : w;
            const double all = group_sum<64>(w);
            w = all > 0.0 ? w / all : 0.0;
        }
        if (lane < K) {
            a.idx[row * K + lane] = mine;
            a.vals[row * K + lane] = (float)(w * (double)a.scale);
        }
    }
}

template <typename T, int R>
__global__ __launch_bounds__(RT_BLOCK) void route_bwd_rows(const RouteRows a) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int E = a.E, K = a.K;
    const double inf = __builtin_inf();
    for (int64_t row = (int64_t)blockIdx.x * RT_WAVES + wv; row < a.N;
         row += (int64_t)gridDim.x * RT_WAVES) {
        const T* xr = static_cast<const T*>(a.x) + row * E;
        T* dr = static_cast<T*>(a.dx) + row * E;
        const int e0 = lane < K ? a.idx[row * K + lane] : -1;
        const bool in = e0 >= 0 && e0 < E;
        const double g = in ? (double)a.dvals[row * K + lane] * (double)a.scale : 0.0;
        const double xc = in ? (double)load1(xr + e0) : -inf;
        double d[R];
#pragma unroll
        for (int j = 0; j < R; ++j) d[j] = 0.0;
        // the gradient of the chosen logits, by place
        double own = 0.0, dot = 0.0, mx = 0.0, rsum = 0.0;
        const bool dense = !a.sigmoid && !a.renorm && __any(in);
        float x[R];
        if (dense) {
            float m = -__builtin_inff();
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int e = j * 64 + lane;
                x[j] = e < E ? load1(xr + e) : -__builtin_inff();
                m = fmaxf(m, x[j]);
            }
            mx = (double)group_max<64>(m);
#pragma unroll
            for (int j = 0; j < R; ++j) {
                d[j] = exp2_wide(((double)x[j] - mx) * kLog2eD);
                sum += d[j];
            }
            rsum = 1.0 / group_sum<64>(sum);
            own = exp2_wide((xc - mx) * kLog2eD) * rsum;
            dot = group_sum<64>(in ? g * own : 0.0);
            own = g * own;
#pragma unroll
            for (int j = 0; j < R; ++j) d[j] = -d[j] * rsum * dot;
        } else if (a.renorm) {
            const double z = !in ? -inf : a.sigmoid ? __builtin_fmin(xc, 0.0) : xc;
            const double zm = (double)group_max<64>((float)z);
            const double e = exp2_wide(-__builtin_fabs(xc) * kLog2eD);
            double p = exp2_wide((z - zm) * kLog2eD);
            if (a.sigmoid) p /= 1.0 + e;
            p = in ? p : 0.0;
            const double all = group_sum<64>(p);
            p = all > 0.0 ? p / all : 0.0;
            dot = group_sum<64>(p * g);
            own = p * (g - dot);
            if (a.sigmoid) own *= (xc >= 0.0 ? e : 1.0) / (1.0 + e);
        } else if (a.sigmoid) {
            const double e = exp2_wide(-__builtin_fabs(xc) * kLog2eD);
            own = g * e / ((1.0 + e) * (1.0 + e));
        }
        // places to experts
        for (int i = 0; i < K; ++i) {
            const int e = __shfl(in ? e0 : -1, i);
            const double v = __shfl(own, i);
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (e == j * 64 + lane) d[j] += v;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int e = j * 64 + lane;
            if (e < E) store1(dr + e, (float)d[j]);
        }
    }
}

template <typename T, bool BWD>
hipError_t launch_route_t(const RouteRows& a, hipStream_t st) {
    const int64_t want = (a.N + RT_WAVES - 1) / RT_WAVES;
    const unsigned blocks = (unsigned)(want < (1 << 20) ? want : 1 << 20);
    const int r = (a.E + 63) / 64;
#define OSM_ROUTE(R)                                                                            \
    do {                                                                                        \
        if constexpr (BWD)                                                                      \
            hipLaunchKernelGGL((route_bwd_rows<T, R>), dim3(blocks), dim3(RT_BLOCK), 0, st, a); \
        else                                                                                    \
            hipLaunchKernelGGL((route_rows<T, R>), dim3(blocks), dim3(RT_BLOCK), 0, st, a);     \
    } while (0)
    if (r <= 1) OSM_ROUTE(1);
    else if (r <= 2) OSM_ROUTE(2);
    else if (r <= 4) OSM_ROUTE(4);
    else if (r <= 8) OSM_ROUTE(8);
    else OSM_ROUTE(16);
#undef OSM_ROUTE
    return hipGetLastError();
}

hipError_t launch_route_fwd(const RouteRows& a, int dtype, hipStream_t st) {
    return dtype == 1 ? launch_route_t<bf16_t, false>(a, st) : launch_route_t<float, false>(a, st);
}

hipError_t launch_route_bwd(const RouteRows& a, int dtype, hipStream_t st) {
    return dtype == 1 ? launch_route_t<bf16_t, true>(a, st) : launch_route_t<float, true>(a, st);
}

}  // namespace osm
