// Routing tokens to experts, and the gradient of the weights.
//
// Forward, a row of E logits x: scores s = softmax(x) or 1 / (1 + e^-x); experts
// are ranked by c = s + bias, or by x itself without a bias (both scores
// increase with x); with groups, each group of E / G experts is ranked by its best
// c, or the sum of its two best (of s without a bias), and only the best top_groups
// are searched; the K largest c, ties to the lower index, give the experts, and
// their s the weights (renormalised to sum 1 if asked, times scale).  Renormalised
// weights are taken from the chosen logits alone, relative to the largest, so they do
// not underflow together.
//
// The choice is that of binary64 scores: a bias brings experts close together, and a
// choice must not depend on the order of a sum.  It is made on binary32 c first.  Of
// those drawn, the ones that are closer than their errors are ranked again in binary64;
// experts are drawn past the K-th until the next one is clearly behind it.  A row whose
// groups are that close on the two sides of the line, or that has more such experts
// than lanes, is done again in binary64 as a whole.  (256 sigmoid scores, 8 taken:
// 3 of 1000 rows have a close pair.)  Where x itself ranks the experts the first choice
// is exact.
//
// A row is taken by LANES lanes, R experts a lane.  Each lane sorts its own, and the K
// are drawn one by one, the largest head first: a 32-bit maximum over the lanes a draw.
//
// Backward, with g the gradient of the K weights and p = weights / scale:
//   softmax, renormalised:  dx_i = scale p_i (g_i - sum_j g_j p_j) at the chosen
//   softmax:                dx_e = scale s_e (g_e - sum_j g_j s_j), everywhere
//   sigmoid, renormalised:  dx_i = scale p_i (g_i - sum_j g_j p_j) (1 - s_i)
//   sigmoid:                dx_i = scale g_i s_i (1 - s_i)
// and 0 elsewhere.  The choice itself has no gradient, and neither has the bias.
//
// What bounds them: 16384 x 256 binary32 sigmoid with a bias and groups takes 25 to 28 us, the
// 17 MB alone 2.6: 640 vector instructions a row and the draws' dependent steps, at four
// wavefronts a SIMD (more of them spill: 34 to 42 us).  Without scores 10007 x 160 bfloat16
// has 475 a row (10.8 us).  The gradient of the first batch, 10.5 us, is 62% of a large
// copy's rate (its 34 MB 6.5).  Calls of some thousand logits are a launch, 3.3 to 4.0 us.
#include "wide.hpp"
#include "kernels.h"

namespace osm {

constexpr int RT_BLOCK = 256;
constexpr int RT_WAVES = RT_BLOCK / 64;

// 1 / d for 1/2 <= d <= 64: the hardware's estimate, to 2^-23, and two Newton steps (each
// squares the error).
__device__ __forceinline__ double reciprocal(double d) {
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    return __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
}

// e^-|x|
__device__ __forceinline__ double exp_minus_abs(double x) {
    return exp2_wide(-__builtin_fabs(x) * kLog2eD);
}

__device__ __forceinline__ double sigmoid_wide(double x) {
    const double e = exp_minus_abs(x), r = reciprocal(1.0 + e);
    return x >= 0.0 ? r : e * r;
}

// Largest distance of a binary32 c = s + bias from the exact one, |bias| <= bmax.  s is at
// most 1: the hardware's 2^t and reciprocal are off by 2^-23 of their value each, the
// rounding of t adds |t| s 2^-23 < 2^-23 (a sigmoid a quarter of both: in all under
// 2^-21); the sum of a softmax adds as much as its terms and 2^-24 for each of at most
// 22 additions (under 2^-19).  The sum with the bias rounds c.
__device__ __forceinline__ float score_error(bool sigmoid, float bmax) {
    return (sigmoid ? 0x1p-20f : 0x1p-18f) + 0x1p-23f * (1.0f + bmax);
}

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

// Sorts a lane's keys, which differ, largest first: Batcher's odd-even merge network.
template <int R>
__device__ __forceinline__ void sort_lane(uint64_t (&k)[R]) {
#pragma unroll
    for (int p = 1; p < R; p *= 2) {
#pragma unroll
        for (int q = p; q >= 1; q /= 2) {
#pragma unroll
            for (int j = q % p; j + q < R; j += 2 * q) {
#pragma unroll
                for (int i = 0; i < q; ++i) {
                    if (i + j + q < R && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                        const uint64_t a = k[i + j], b = k[i + j + q];
                        const bool swap = b > a;
                        k[i + j] = swap ? b : a;
                        k[i + j + q] = swap ? a : b;
                    }
                }
            }
        }
    }
}

// Place of a number in LDS where rows of 32 are walked side by side: a free one after each
// 32 puts them into different banks.
constexpr __device__ __forceinline__ int padded(int i) { return i + i / 32; }

template <int LANES>
__device__ __forceinline__ float team_min(float v) {
    return -group_max<LANES>(-v);
}

// A row's experts in binary64, by the whole wavefront: the K best one after the other,
// each the first in the order (c, index) behind the one before.  rk: E ranks, the
// order of c (0 for an expert that cannot be chosen).
template <typename T>
__device__ __forceinline__ void exact_row(const RouteRows& a, const T* xr, float mx, uint64_t* rk,
                                          int* ch) {
    const int lane = threadIdx.x & 63;
    const int E = a.E, G = a.groups;
    double sum = 0.0;
    for (int e = lane; e < E; e += 64) {
        const double x = (double)load1(xr + e);
        const double s = a.sigmoid ? sigmoid_wide(x) : exp2_wide((x - (double)mx) * kLog2eD);
        rk[e] = __builtin_bit_cast(uint64_t, s);
        sum += s;
    }
    const double rsum = a.sigmoid ? 1.0 : 1.0 / group_sum<64>(sum);
    for (int e = lane; e < E; e += 64) {
        const float b = a.bias ? a.bias[e] : 0.0f;
        const bool may = load1(xr + e) > -__builtin_inff() && b > -__builtin_inff();
        const double s = __builtin_bit_cast(double, rk[e]) * rsum;
        rk[e] = may ? order_key(s + (double)b) : 0;
    }
    wave_sync();
    if (G > 1) {
        const int gs = E / G;
        int per = 64;
        while (per * G > 64) per >>= 1;
        const int g = lane / per;
        uint64_t best = 0, second = 0;
        if (g < G) {
            for (int i = lane % per; i < gs; i += per) {
                const uint64_t k = rk[g * gs + i];
                second = k > best ? best : k > second ? k : second;
                best = k > best ? k : best;
            }
        }
        for (int d = 1; d < per; d *= 2) {
            const uint64_t k = __shfl_xor(best, d), k2 = __shfl_xor(second, d);
            const uint64_t lo = k > best ? best : k, hi2 = k2 > second ? k2 : second;
            best = k > best ? k : best;
            second = lo > hi2 ? lo : hi2;
        }
        if (a.group_top == 2 && second != 0)
            best = order_key(order_value64(best) + order_value64(second));
        int ahead = 0;
        for (int o = 0; o < G; ++o) {
            const uint64_t k = lane_value(best, o * per);
            ahead += k > best || (k == best && o < g);
        }
        if (g < G && ahead >= a.top_groups)
            for (int i = lane % per; i < gs; i += per) rk[g * gs + i] = 0;
        wave_sync();
    }
    if (!a.bias) {  // the experts of the kept groups by x again
        for (int e = lane; e < E; e += 64)
            rk[e] = rk[e] != 0 ? (uint64_t)order_key(load1(xr + e)) << 32 : 0;
        wave_sync();
    }
    for (int i = 0; i < a.K; ++i) {
        uint64_t best = 0;
        int at = 0;
        for (int e = lane; e < E; e += 64) {
            const uint64_t k = rk[e];
            at = k > best ? e : at;
            best = k > best ? k : best;
        }
        const uint64_t top = group_max<64>(best);
        const uint32_t e = ~group_max<64>(best == top ? ~(uint32_t)at : 0u);
        if (lane == 0) {
            ch[i] = top != 0 ? (int)e : -1;
            rk[e] = 0;
        }
        wave_sync();
    }
}

// SCORES: with a bias, or groups ranked by the sum of their two best; without them x is
// what ranks the experts.
template <typename T, int LANES, int R, int VEC, bool SCORES>
__global__ __launch_bounds__(RT_BLOCK) void route_rows(const RouteRows a) {
    constexpr int ROWS = 64 / LANES;  // of a wavefront
    const float ninf = -__builtin_inff();
    __shared__ uint64_t ranks[RT_WAVES][SCORES ? 64 * R : (ROWS * padded(LANES * R) + 1) / 2];
    __shared__ float best_of[RT_WAVES][64];
    __shared__ int chosen[RT_WAVES][64];
    const int lane = threadIdx.x % LANES, wv = threadIdx.x >> 6, team = (threadIdx.x & 63) / LANES;
    const int E = a.E, K = a.K, G = a.groups;
    float* const hc = reinterpret_cast<float*>(ranks[wv]) + team * padded(LANES * R);
    float* const go = best_of[wv] + team * LANES;
    int* const ch = chosen[wv] + team * LANES;
    const bool sums = SCORES && G > 1 && a.group_top == 2;
    const bool biased = SCORES && a.bias;
    const int gs = G > 1 ? E / G : E;
    const float rgs = 1.0f / (float)gs;
    int per = LANES;  // lanes that look at a group
    while (per * G > LANES) per >>= 1;
    for (int64_t row0 = ((int64_t)blockIdx.x * RT_WAVES + wv) * ROWS; row0 < a.N;
         row0 += (int64_t)gridDim.x * RT_WAVES * ROWS) {
        const int64_t row = row0 + team;
        const bool live = row < a.N;
        const T* xr = static_cast<const T*>(a.x) + (live ? row : 0) * E;
        float x[R], c[R];
        load_experts<T, LANES, R, VEC>(xr, E, live, lane, x);
        float mx = x[0];
#pragma unroll
        for (int j = 1; j < R; ++j) mx = __builtin_elementwise_maximum(mx, x[j]);
        mx = team_maximum<LANES>(mx);
        const bool bad = !(mx < __builtin_inff());
        const bool some = !bad && mx > ninf;
        double rsum = 1.0;  // of the exact scores
        if (!a.sigmoid && !a.renorm) {
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                sum += exp2_wide(((double)x[j] - (double)mx) * kLog2eD);
            }
            rsum = 1.0 / group_sum<LANES>(sum);
        }
        float error = 0.0f;
        if constexpr (SCORES) {
            float rs = 1.0f, bmax = 0.0f;
            if (a.sigmoid) {
#pragma unroll
                for (int j = 0; j < R; ++j)
                    c[j] = __builtin_amdgcn_rcpf(1.0f + exp2_hw(-x[j] * kLog2e));
            } else {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    c[j] = exp2_hw((x[j] - mx) * kLog2e);
                    sum += c[j];
                }
                rs = 1.0f / group_sum<LANES>(sum);
            }
            float b[R];
            if (biased) {
                load_experts<float, LANES, R, VEC>(a.bias, E, true, lane, b);
            } else {
#pragma unroll
                for (int j = 0; j < R; ++j) b[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const float m = __builtin_fabsf(b[j]);
                bmax = m < __builtin_inff() ? fmaxf(bmax, m) : bmax;
                // (a NaN bias: no)
                const bool may = some && x[j] > ninf && b[j] > ninf;
                c[j] = may ? __builtin_fmaf(c[j], rs, b[j]) : ninf;
            }
            error = score_error(a.sigmoid, biased ? group_max<LANES>(bmax) : 0.0f);
        } else {
#pragma unroll
            for (int j = 0; j < R; ++j) c[j] = some ? x[j] : ninf;
        }
        bool again = false;  // a line that binary32 does not decide
        if (G > 1) {
#pragma unroll
            for (int j = 0; j < R; ++j) hc[padded(expert<LANES, VEC>(lane, j))] = c[j];
            wave_sync();
            const int g = lane / per;
            float best = ninf, second = ninf;
            if (g < G) {
                for (int i = lane % per; i < gs; i += per) {
                    const float v = hc[padded(g * gs + i)];
                    second = __builtin_amdgcn_fmed3f(v, best, second);
                    best = fmaxf(best, v);
                }
            }
            for (int d = 1; d < per; d *= 2) {
                const float v = __shfl_xor(best, d), v2 = __shfl_xor(second, d);
                second = fmaxf(fminf(best, v), fmaxf(second, v2));
                best = fmaxf(best, v);
            }
            if (sums && best > ninf) {
                // a sum that leaves binary32 (two biases of the type's lowest value) is not
                // that of a group without experts: the largest numbers stand for all beyond
                // them, and groups that are equal here are ranked again in binary64
                constexpr float most = __FLT_MAX__;
                best = __builtin_amdgcn_fmed3f(second > ninf ? best + second : best, -most, most);
            }
            if (g < G && lane % per == 0) go[g] = best;
            wave_sync();
            int ahead = 0;
            for (int o = 0; o < G; ++o) {
                const float v = go[o];
                ahead += v > best || (v == best && o < g);
            }
            const bool stays = g < G && ahead < a.top_groups;
            const uint64_t keep = __ballot(stays);
            if constexpr (SCORES) {
                const float low = team_min<LANES>(stays ? best : __builtin_inff());
                const float high = group_max<LANES>(g < G && !stays ? best : ninf);
                again = high > ninf && low < __builtin_inff() && !(low - high > 4.0f * error);
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                // (the quotient of numbers up to 1024 by a reciprocal: half a unit is far
                // more than its error)
                const int e = expert<LANES, VEC>(lane, j);
                const int ge = (int)(((float)(e < E ? e : 0) + 0.5f) * rgs);
                if (!(keep >> (ge * per + team * LANES) & 1)) c[j] = ninf;
            }
            if (sums && !biased) {  // the experts of the kept groups by x again
#pragma unroll
                for (int j = 0; j < R; ++j) c[j] = c[j] > ninf ? x[j] : ninf;
            }
        }
        ch[lane] = -1;
        wave_sync();
        // keys: the order of c, then the lower index; 0 for what cannot be chosen
        uint64_t k[R];
#pragma unroll
        for (int j = 0; j < R; ++j)
            k[j] = c[j] > ninf ? (uint64_t)order_key(c[j]) << 32 |
                                     (uint32_t)~(uint32_t)expert<LANES, VEC>(lane, j)
                               : 0;
        sort_lane(k);
        float before = __builtin_inff();
        bool close = false, open = true;  // open: the next one may still matter
        int drawn = 0;
        for (int i = 0;; ++i) {
            if (!biased && i == K) break;
            const uint32_t hi = (uint32_t)(k[0] >> 32), top = group_max<LANES>(hi);
            open = open && top != 0;
            if (biased) {
                // past the K-th, those that are too close to the one before to be behind it
                const float v = order_value(top);
                const bool near = !(before - v > 2.0f * error);  // (equal ones among them)
                open = open && (i < K || near);
                close = close || (open && i > 0 && near);
                before = v;
                if (i == LANES) {  // (no lane for another)
                    again = again || open;
                    break;
                }
            }
            const int teams = __popcll(__ballot(open)) / LANES;
            if (teams == 0) break;
            bool win = open && hi == top;
            if (__popcll(__ballot(win)) != teams) {
                const uint32_t lo = group_max<LANES>(win ? (uint32_t)k[0] : 0u);
                win = win && (uint32_t)k[0] == lo;
            }
            drawn += open;
            if (win) {
                ch[i] = (int)~(uint32_t)k[0];
#pragma unroll
                for (int j = 0; j + 1 < R; ++j) k[j] = k[j + 1];
                k[R - 1] = 0;
            }
        }
        wave_sync();
        int pick = ch[lane];
        if constexpr (SCORES) {
            if (__ballot(close && live) != 0) {
                // the drawn ones by their exact c, and by the index where that is equal
                double rs = 1.0;
                if (!a.sigmoid) {
                    double sum = 0.0;
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        sum += exp2_wide(((double)x[j] - (double)mx) * kLog2eD);
                            }
                    rs = 1.0 / group_sum<LANES>(sum);
                }
                uint64_t mine = 0;
                if (pick >= 0) {
                    const double xp = (double)load1(xr + pick);
                    const double s = a.sigmoid ? sigmoid_wide(xp)
                                               : exp2_wide((xp - (double)mx) * kLog2eD) * rs;
                    mine = order_key(s + (double)a.bias[pick]);
                }
                uint64_t* const rk = ranks[wv] + team * LANES;
                rk[lane] = mine;
                wave_sync();
                int ahead = 0;
                const int most = (int)group_max<64>((uint32_t)drawn);
                for (int i = 0; i < most; ++i) {
                    const uint64_t o = rk[i];
                    ahead += o > mine || (o == mine && ch[i] < pick);
                }
                wave_sync();
                if (pick >= 0) ch[ahead] = pick;
                wave_sync();
                pick = ch[lane];
            }
            uint64_t rows = __ballot(again && some && live);
            if (rows) {
                while (rows) {  // (uniform: a row of the wavefront at a time)
                    const int r = __builtin_ctzll(rows) / LANES;
                    rows = LANES == 64 ? 0
                                       : rows & ~(((1ull << (LANES & 63)) - 1) << (r * LANES));
                    wave_sync();
                    exact_row(a, static_cast<const T*>(a.x) + (row0 + r) * E,
                              lane_value(mx, r * LANES), ranks[wv], chosen[wv] + r * LANES);
                }
                wave_sync();
                pick = ch[lane];
            }
        }
        wave_sync();
        // weights: lane i has the i-th expert
        if (lane >= K) pick = -1;
        const double xp = pick >= 0 ? (double)load1(xr + pick) : -__builtin_inf();
        double w = 0.0;
        if (a.renorm) {
            // relative to the largest chosen one: e^x, or e^min(x, 0) / (1 + e^-|x|)
            const double z = a.sigmoid ? __builtin_fmin(xp, 0.0) : xp;
            const double zm = (double)team_maximum<LANES>((float)z);
            w = exp2_wide((z - zm) * kLog2eD);
            if (a.sigmoid) w *= reciprocal(1.0 + exp_minus_abs(xp));
            w = pick >= 0 ? w : 0.0;
            const double all = group_sum<LANES>(w);  // at least 1/2, if any
            w = all > 0.0 ? w * reciprocal(all) : 0.0;
        } else if (pick >= 0) {
            w = a.sigmoid ? sigmoid_wide(xp) : exp2_wide((xp - (double)mx) * kLog2eD) * rsum;
        }
        if (live && lane < K) {
            a.idx[row * K + lane] = pick;
            a.vals[row * K + lane] = bad ? __builtin_nanf("") : (float)(w * (double)a.scale);
        }
    }
}

// The gradient.  A row by LANES lanes, R experts a lane; lane i also has place i.
template <typename T, int LANES, int R, int VEC>
__global__ __launch_bounds__(RT_BLOCK) void route_bwd_rows(const RouteRows a) {
    constexpr int ROWS = 64 / LANES;
    __shared__ double owns[RT_WAVES][64];
    __shared__ int places[RT_WAVES][64];
    __shared__ __align__(16) int place_of[RT_WAVES][64 * R];
    const int lane = threadIdx.x % LANES, wv = threadIdx.x >> 6, team = (threadIdx.x & 63) / LANES;
    const int E = a.E, K = a.K;
    double* const so = owns[wv] + team * LANES;
    int* const sp = places[wv] + team * LANES;
    int* const po = place_of[wv] + team * LANES * R;
    const bool dense = !a.sigmoid && !a.renorm;
    for (int64_t row0 = ((int64_t)blockIdx.x * RT_WAVES + wv) * ROWS; row0 < a.N;
         row0 += (int64_t)gridDim.x * RT_WAVES * ROWS) {
        const int64_t row = row0 + team;
        const bool live = row < a.N;
        const T* xr = static_cast<const T*>(a.x) + (live ? row : 0) * E;
        float x[R];
        if (dense) load_experts<T, LANES, R, VEC>(xr, E, live, lane, x);
        const int e0 = live && lane < K ? a.idx[row * K + lane] : -1;
        const bool in = e0 >= 0 && e0 < E;
        const double g = in ? (double)a.dvals[row * K + lane] * (double)a.scale : 0.0;
        const double xc = in ? (double)load1(xr + e0) : -__builtin_inf();
        double d[R], own;
        if (dense) {
            float m = x[0];
#pragma unroll
            for (int j = 1; j < R; ++j) m = __builtin_elementwise_maximum(m, x[j]);
            const double mx = (double)team_maximum<LANES>(m);
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                d[j] = exp2_wide(((double)x[j] - mx) * kLog2eD);
                sum += d[j];
            }
            const double rsum = 1.0 / group_sum<LANES>(sum);
            own = g * (exp2_wide((xc - mx) * kLog2eD) * rsum);
            // (a row without any place, whatever it holds, has no gradient)
            const uint64_t who = __ballot(in);
            const uint64_t row_mask = LANES == 64 ? ~0ull
                                                  : ((1ull << (LANES & 63)) - 1) << (team * LANES);
            const bool any = (who & row_mask) != 0;
            const double dot = group_sum<LANES>(in ? own : 0.0) * rsum;
#pragma unroll
            for (int j = 0; j < R; ++j) d[j] = any ? -d[j] * dot : 0.0;
        } else {
#pragma unroll
            for (int j = 0; j < R; ++j) d[j] = 0.0;
            const double e = exp_minus_abs(xc), f = reciprocal(1.0 + e);
            if (a.renorm) {
                const double z = a.sigmoid && xc > 0.0 ? 0.0 : xc;  // (NaN stays)
                const double zm = (double)team_maximum<LANES>(in ? (float)z : -__builtin_inff());
                double p = exp2_wide((z - zm) * kLog2eD);
                if (a.sigmoid) p *= f;
                p = in ? p : 0.0;
                const double all = group_sum<LANES>(p);
                p = all > 0.0 ? p / all : 0.0;
                own = p * (g - group_sum<LANES>(p * g));
                // a chosen NaN (or the softmax of +inf) leaves no weight a number
                if (!(zm < __builtin_inf())) own = __builtin_nan("");
                if (a.sigmoid) own *= (xc >= 0.0 ? e : 1.0) * f;
            } else {
                own = xc == xc ? g * e * f * f : xc;
            }
        }
        // places to experts: each expert finds the place that it has, if any
        so[lane] = own;
        if constexpr (VEC == 1) {
#pragma unroll
            for (int j = 0; j < R; ++j) po[expert<LANES, VEC>(lane, j)] = -1;
        } else {
#pragma unroll
            for (int j = 0; j < R; j += 4)
                *reinterpret_cast<int4*>(po + expert<LANES, VEC>(lane, j)) = int4{-1, -1, -1, -1};
        }
        wave_sync();
        if (in) po[e0] = lane;
        wave_sync();
        if (__any(in && po[e0] != lane)) {  // an expert twice: all places, in their order
            sp[lane] = in ? e0 : -1;
            wave_sync();
            for (int i = 0; i < K; ++i) {
                const int e = sp[i];
                const double v = so[i];
#pragma unroll
                for (int j = 0; j < R; ++j)
                    if (e == expert<LANES, VEC>(lane, j)) d[j] += v;
            }
        } else {
            int p[R];
            if constexpr (VEC == 1) {
#pragma unroll
                for (int j = 0; j < R; ++j) p[j] = po[expert<LANES, VEC>(lane, j)];
            } else {
#pragma unroll
                for (int j = 0; j < R; j += 4) {
                    const int4 q = *reinterpret_cast<const int4*>(po + expert<LANES, VEC>(lane, j));
                    p[j] = q.x, p[j + 1] = q.y, p[j + 2] = q.z, p[j + 3] = q.w;
                }
            }
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (p[j] >= 0) d[j] += so[p[j]];
        }
        wave_sync();
        if (!live) continue;
        T* dr = static_cast<T*>(a.dx) + row * E;
        if constexpr (VEC == 1) {
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (j * LANES + lane < E) store1(dr + j * LANES + lane, (float)d[j]);
        } else {
#pragma unroll
            for (int j = 0; j < R; j += 4) {
                const int e = expert<LANES, VEC>(lane, j);
                if (e >= E) continue;
                if constexpr (sizeof(T) == 4)
                    *reinterpret_cast<f32x4*>(dr + e) =
                        f32x4{(float)d[j], (float)d[j + 1], (float)d[j + 2], (float)d[j + 3]};
                else
                    *reinterpret_cast<uint2*>(dr + e) =
                        uint2{pack_bf16x2((float)d[j], (float)d[j + 1]),
                              pack_bf16x2((float)d[j + 2], (float)d[j + 3])};
            }
        }
    }
}

// Lanes of a row: enough for its K places and its groups, and for its experts at
// `each` a lane or few more.
static int route_lanes(const RouteRows& a, int each) {  // (each <= 8: launch_route_l)
    int lanes = 8;
    while (lanes < 64 && (lanes < a.K || lanes < a.groups || lanes * each < a.E)) lanes *= 2;
    return lanes;
}

template <typename T, bool BWD, int LANES, int R, int VEC>
hipError_t launch_route_r(const RouteRows& a, unsigned blocks, hipStream_t st) {
    if constexpr (BWD)
        hipLaunchKernelGGL((route_bwd_rows<T, LANES, R, VEC>), dim3(blocks), dim3(RT_BLOCK), 0, st,
                           a);
    else if (a.bias || (a.groups > 1 && a.group_top == 2))
        hipLaunchKernelGGL((route_rows<T, LANES, R, VEC, true>), dim3(blocks), dim3(RT_BLOCK), 0,
                           st, a);
    else
        hipLaunchKernelGGL((route_rows<T, LANES, R, VEC, false>), dim3(blocks), dim3(RT_BLOCK), 0,
                           st, a);
    return hipGetLastError();
}

template <typename T, bool BWD, int LANES, int VEC>
hipError_t launch_route_l(const RouteRows& a, hipStream_t st) {
    const int64_t want = (a.N + RT_WAVES * (64 / LANES) - 1) / (RT_WAVES * (64 / LANES));
    const int64_t most = (int64_t)a.cus * (BWD ? 5 : 4);
    const unsigned blocks = (unsigned)(want < most ? want : most);
    const int r = (a.E + LANES - 1) / LANES;
    if constexpr (VEC == 1) {
        if (r <= 1) return launch_route_r<T, BWD, LANES, 1, VEC>(a, blocks, st);
        if (r <= 2) return launch_route_r<T, BWD, LANES, 2, VEC>(a, blocks, st);
    }
    if (r <= 4) return launch_route_r<T, BWD, LANES, 4, VEC>(a, blocks, st);
    if constexpr (LANES < 64) return launch_route_r<T, BWD, LANES, 8, VEC>(a, blocks, st);
    if (r <= 8) return launch_route_r<T, BWD, LANES, 8, VEC>(a, blocks, st);
    return launch_route_r<T, BWD, LANES, 16, VEC>(a, blocks, st);
}

template <typename T, bool BWD>
hipError_t launch_route_t(const RouteRows& a, hipStream_t st) {
    // four neighbours at a time where every row (and the bias) allows it
    const uintptr_t at = (uintptr_t)a.x | (BWD ? (uintptr_t)a.dx : 0);
    const bool vec = a.E % 4 == 0 && at % (4 * sizeof(T)) == 0 && (uintptr_t)a.bias % 16 == 0 &&
                     a.E >= 32;
#define OSM_LANES(L) \
    return vec ? launch_route_l<T, BWD, L, 4>(a, st) : launch_route_l<T, BWD, L, 1>(a, st)
    // Eight experts a lane once the batch fills the chip: the steps over the lanes then serve
    // twice as many rows.  Else four.  us with eight and four, binary32 sigmoid with a bias
    // and groups: 1024 x 256 8.8 and 8.0, 2048 x 256 9.4 and 9.5, 4096 x 128 9.7 and 9.7,
    // 4096 x 160 9.2 and 11.1, 4096 x 256 10.7 and 12.7, 16384 x 256 29 and 42; softmax
    // without scores 2048 x 256 6.7 and 6.0, 4096 x 160 6.7 and 7.0, 16384 x 256 16 and 22;
    // the dense gradient 1024 x 256 4.0 and 3.7, 4096 x 160 4.8 and 4.9, 16384 x 256 10.2
    // and 13.4.  (From 257 experts on both are the same.)
    switch (route_lanes(a, a.N * a.E > (int64_t)a.cus * 2048 ? 8 : 4)) {
        case 8: OSM_LANES(8);
        case 16: OSM_LANES(16);
        case 32: OSM_LANES(32);
        default: OSM_LANES(64);
    }
#undef OSM_LANES
}

hipError_t launch_route_fwd(const RouteRows& a, int dtype, hipStream_t st) {
    return dtype == 1 ? launch_route_t<bf16_t, false>(a, st) : launch_route_t<float, false>(a, st);
}

hipError_t launch_route_bwd(const RouteRows& a, int dtype, hipStream_t st) {
    return dtype == 1 ? launch_route_t<bf16_t, true>(a, st) : launch_route_t<float, true>(a, st);
}

}  // namespace osm
