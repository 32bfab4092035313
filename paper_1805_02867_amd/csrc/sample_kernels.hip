// Sampling a token of each row: temperature, top-k, top-p and min-p, with the
// random number given.
//
// With m the row's maximum, the weights are w_j = 2^{(x_j - m) log2(e) / T}.  Each
// filter keeps a prefix of the order "x descending, index ascending", so all
// of them together are one cut in that order, held as the 64-bit key
// (ordered x) << 32 | ~index of the last kept element:
//   top-k  the k-th element;
//   top-p  the first element at which the sum of weights, in that order and over
//          what top-k kept, reaches p times the whole;
//   min-p  the last element with w_j >= min_p (a test on the weight).
// Nothing is sorted: a cut is found by histograms over the keys, each round
// over the bin in which the count (top-k) or the mass (top-p) passes its target.
// Masses in the histograms are weights in fixed point, whose sums do not depend
// on the order of the atomic additions.
//
// The token is the first kept one, in index order, at which the running sum
// passes u times the sum of the kept weights.
//
// Weights and sums are binary64: in binary32 the sums of 10^5 weights are off by
// more than the distance between the borders they put on [0, 1), and the token
// would depend on the order of the additions.
#include "wide.hpp"
#include "kernels.h"

namespace osm {

constexpr int SM_BLOCK = 512;
constexpr int SM_WAVES = SM_BLOCK / 64;
constexpr int SM_LOG_BINS = 10;
constexpr int SM_BINS = 1 << SM_LOG_BINS;
static_assert(SM_BINS == 2 * SM_BLOCK, "two bins a thread");

struct SampleSmem {
    union {
        uint64_t bins[SM_BINS];
        double seg[SM_BINS];
    };
    uint64_t wave64[SM_WAVES];
    double waved[SM_WAVES];
    uint32_t wave32[SM_WAVES];
    int flag[SM_WAVES];
    int found;
    uint64_t above, here;
    double base;
};

// What a row asks for.
struct Rule {
    bool greedy;
    double c;       // log2(e) / T
    int64_t k;      // elements that top-k keeps (0: all)
    double p, q, u;
};

__device__ __forceinline__ Rule row_rule(const SampleRows& a, int64_t row) {
    const float T = a.temperature ? a.temperature[row] : a.temperature_all;
    const int32_t k = a.top_k ? a.top_k[row] : a.top_k_all;
    const float p = a.top_p ? a.top_p[row] : a.top_p_all;
    const float q = a.min_p ? a.min_p[row] : a.min_p_all;
    const float u = a.u[row];
    Rule r;
    r.greedy = !(T > 0.0f);
    r.c = kLog2eD / (double)T;
    r.k = k > 0 && k < a.V ? k : 0;
    r.p = p < 1.0f ? (double)p : 1.0;  // (NaN: off)
    r.q = q > 0.0f ? __builtin_fmin((double)q, 1.0) : 0.0;
    r.u = u > 0.0f ? __builtin_fmin((double)u, 1.0) : 0.0;
    return r;
}

// w of x; 0 at -inf, whatever c.
__device__ __forceinline__ double weight(float x, double m, double c) {
    return exp2_wide(((double)x - m) * c);
}

// A weight in fixed point, to nearest.
__device__ __forceinline__ uint64_t fixed(double w, double scale) {
    return (uint64_t)__builtin_fma(w, scale, 0.5);
}

template <typename T>
struct RowSource {
    const T* x;
    int64_t n;
    __device__ __forceinline__ float value(int64_t i) const { return load1(x + i); }
};

// The bin in which the running sum over sm.bins reaches `target`, with the sum
// before it: results in sm.found, sm.above (which starts at `above`) and sm.here.
// p >= 0: the target is the part p of the bins' sum, at least 1, and is returned.
__device__ __forceinline__ uint64_t find_bin(SampleSmem& sm, uint64_t above, uint64_t target,
                                             double p) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const uint64_t a = sm.bins[2 * tid], b = sm.bins[2 * tid + 1];
    const uint64_t incl = wave_scan(a + b);
    if (lane == 63) sm.wave64[wv] = incl;
    __syncthreads();
    uint64_t before = above, total = above;
#pragma unroll
    for (int w = 0; w < SM_WAVES; ++w) {
        if (w < wv) before += sm.wave64[w];
        total += sm.wave64[w];
    }
    if (p >= 0.0) {
        const double want = __builtin_ceil(p * (double)total);
        target = want >= 1.0 ? (uint64_t)want : 1;
        target = target < total ? target : total;
    }
    before += incl - a - b;
    if (before < target && target <= before + a) {
        sm.found = 2 * tid;
        sm.above = before;
        sm.here = a;
    } else if (before + a < target && target <= before + a + b) {
        sm.found = 2 * tid + 1;
        sm.above = before + a;
        sm.here = b;
    }
    __syncthreads();
    return target;
}

__device__ __forceinline__ int bin_shift(uint32_t range) {
    const int bits = 32 - __builtin_clz(range | 1u);
    return bits > SM_LOG_BINS ? bits - SM_LOG_BINS : 0;
}

// The cut behind which `target` elements (MASS: the part p of the weights) of
// those at or above `cut` lie.
template <bool MASS, typename Src>
__device__ __forceinline__ uint64_t find_cut(SampleSmem& sm, const Src src, uint32_t lo,
                                             uint32_t hi, uint64_t cut, uint64_t target, double p,
                                             double m, double c, double scale) {
    const int tid = threadIdx.x;
    uint64_t above = 0;
    bool first = MASS;
    for (;;) {  // rounds over values
        const int shift = bin_shift(hi - lo);
        sm.bins[tid] = 0;
        sm.bins[tid + SM_BLOCK] = 0;
        __syncthreads();
        for (int64_t i = tid; i < src.n; i += SM_BLOCK) {
            const float x = src.value(i);
            const uint32_t k = order_key(x);
            if (k < lo || k > hi || ((uint64_t)k << 32 | (uint32_t)~(uint32_t)i) < cut) continue;
            const uint64_t w = MASS ? fixed(weight(x, m, c), scale) : 1;
            atomicAdd((unsigned long long*)&sm.bins[(hi - k) >> shift], (unsigned long long)w);
        }
        __syncthreads();
        target = find_bin(sm, above, target, first ? p : -1.0);
        first = false;
        above = sm.above;
        hi -= (uint32_t)sm.found << shift;
        if (shift == 0) break;
        const uint32_t width = (1u << shift) - 1;
        lo = hi - lo > width ? hi - width : lo;
        __syncthreads();
    }
    // the value is hi; how many of the elements that hold it are kept
    const uint64_t w = MASS ? fixed(weight(order_value(hi), m, c), scale) : 1;
    const uint64_t ties = sm.here / w, need = (target - above + w - 1) / w;
    __syncthreads();
    uint64_t last = (uint64_t)hi << 32;
    if (need < ties) {
        uint32_t ilo = 0, ihi = (uint32_t)(src.n - 1);
        above = 0;
        for (;;) {  // rounds over the indices of the ties
            const int shift = bin_shift(ihi - ilo);
            sm.bins[tid] = 0;
            sm.bins[tid + SM_BLOCK] = 0;
            __syncthreads();
            for (int64_t i = (int64_t)ilo + tid; i <= (int64_t)ihi; i += SM_BLOCK) {
                const uint32_t k = order_key(src.value(i));
                if (k != hi || ((uint64_t)k << 32 | (uint32_t)~(uint32_t)i) < cut) continue;
                atomicAdd((unsigned long long*)&sm.bins[((uint32_t)i - ilo) >> shift], 1ull);
            }
            __syncthreads();
            find_bin(sm, above, need, -1.0);
            above = sm.above;
            ilo += (uint32_t)sm.found << shift;
            __syncthreads();
            if (shift == 0) break;
            const uint32_t width = (1u << shift) - 1;
            ihi = ihi - ilo > width ? ilo + width : ihi;
        }
        last |= (uint32_t)~ilo;
    }
    return last > cut ? last : cut;
}

// One row by the workgroup.
template <typename Src>
__device__ __forceinline__ void sample_row(SampleSmem& sm, const Src src, const Rule r,
                                           float* val, int32_t* idx) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    // the maximum with its lowest index, and whether a NaN or +inf is there
    uint64_t best = 0;
    int bad = 0;
    for (int64_t i = tid; i < src.n; i += SM_BLOCK) {
        const float x = src.value(i);
        bad |= !(x < __builtin_inff());
        const uint64_t k = (uint64_t)order_key(x) << 32 | (uint32_t)~(uint32_t)i;
        best = k > best ? k : best;
    }
    best = group_max<64>(best);
    bad = __any(bad);
    if (lane == 0) {
        sm.wave64[wv] = best;
        sm.flag[wv] = bad;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SM_WAVES; ++w) {
        best = sm.wave64[w] > best ? sm.wave64[w] : best;
        bad |= sm.flag[w];
    }
    __syncthreads();
    const float mx = order_value((uint32_t)(best >> 32));
    if (bad || mx == -__builtin_inff() || r.greedy) {
        if (tid == 0) {
            const bool none = bad || mx == -__builtin_inff();
            *idx = none ? -1 : (int32_t)~(uint32_t)best;
            *val = none ? __builtin_nanf("") : 1.0f;
        }
        return;
    }
    const double m = mx;
    const uint32_t top = (uint32_t)(best >> 32), bottom = order_key(-__builtin_inff());
    uint64_t cut = 0;
    if (r.k) cut = find_cut<false>(sm, src, bottom, top, cut, (uint64_t)r.k, 0.0, m, r.c, 0.0);
    if (r.p < 1.0) {
        // the largest weight is 2^s with n 2^s <= 2^62
        const int s = 62 - (64 - __builtin_clzll((uint64_t)src.n));
        cut = find_cut<true>(sm, src, bottom, top, cut, 0, r.p > 0.0 ? r.p : 0.0, m, r.c,
                             __builtin_ldexp(1.0, s));
    }

    // the token: sums of up to SM_BINS segments of the range, then the segment
    // that the target falls into as the next range
    int64_t a = 0, b = src.n;
    double target = 0.0, total = 0.0;
    bool first = true;
    do {
        int64_t L = (b - a + SM_BINS - 1) / SM_BINS;
        L = (L + 63) / 64 * 64;
        for (int s = wv; s < SM_BINS; s += SM_WAVES) {
            double sum = 0.0;
            const int64_t e = a + (s + 1) * L < b ? a + (s + 1) * L : b;
            for (int64_t i = a + s * L + lane; i < e; i += 64) {
                const float x = src.value(i);
                const double w = weight(x, m, r.c);
                const uint64_t k = (uint64_t)order_key(x) << 32 | (uint32_t)~(uint32_t)i;
                sum += k >= cut && w >= r.q ? w : 0.0;
            }
            sum = group_sum<64>(sum);
            if (lane == 0) sm.seg[s] = sum;
        }
        if (tid == 0) sm.found = SM_BINS;
        __syncthreads();
        const double s0 = sm.seg[2 * tid], s1 = sm.seg[2 * tid + 1];
        const double incl = wave_scan(s0 + s1);
        if (lane == 63) sm.waved[wv] = incl;
        __syncthreads();
        double before = 0.0, all = 0.0;
#pragma unroll
        for (int w = 0; w < SM_WAVES; ++w) {
            if (w < wv) before += sm.waved[w];
            all += sm.waved[w];
        }
        if (first) {
            total = all;
            target = r.u * all;
            first = false;
        }
        const double prev = __shfl_up(incl, 1);
        before += lane ? prev : 0.0;
        // (a last positive segment stands in where rounding leaves the target unreached)
        const bool in0 = s0 > 0.0 && before + s0 > target;
        const bool in1 = s1 > 0.0 && before + s0 + s1 > target;
        if (in0 || in1) atomicMin(&sm.found, in0 ? 2 * tid : 2 * tid + 1);
        __syncthreads();
        int at = sm.found;
        __syncthreads();
        if (at == SM_BINS) {
            if (tid == 0) sm.found = -1;
            __syncthreads();
            if (s1 > 0.0) atomicMax(&sm.found, 2 * tid + 1);
            else if (s0 > 0.0) atomicMax(&sm.found, 2 * tid);
            __syncthreads();
            at = sm.found;
            target = __builtin_inf();
        }
        if (tid == at / 2) sm.base = at & 1 ? before + s0 : before;
        __syncthreads();
        target -= sm.base;
        a += at * L;
        b = a + L < b ? a + L : b;
        __syncthreads();
    } while (b - a > 64);
    if (wv == 0) {
        const int64_t i = a + lane;
        double w = 0.0;
        if (i < b) {
            const float x = src.value(i);
            const uint64_t k = (uint64_t)order_key(x) << 32 | (uint32_t)~(uint32_t)i;
            w = weight(x, m, r.c);
            w = k >= cut && w >= r.q ? w : 0.0;
        }
        const double incl = wave_scan(w);
        const uint64_t some = __ballot(w > 0.0);
        const uint64_t past = __ballot(w > 0.0 && incl > target);
        const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
        if (lane == at) {
            *idx = (int32_t)i;
            *val = (float)(w / total);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(SM_BLOCK) void sample_rows(const SampleRows a) {
    __shared__ SampleSmem sm;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const RowSource<T> src{static_cast<const T*>(a.x) + row * a.ld, a.V};
        sample_row(sm, src, row_rule(a, row), a.vals + row, a.idx + row);
        __syncthreads();
    }
}

hipError_t launch_sample(const SampleRows& a, int dtype, hipStream_t st) {
    // (a launch takes fewer than 2^32 threads: further rows by the same workgroups)
    const unsigned blocks = (unsigned)(a.N < (1 << 22) ? a.N : 1 << 22);
    if (dtype == 1)
        hipLaunchKernelGGL(sample_rows<bf16_t>, dim3(blocks), dim3(SM_BLOCK), 0, st, a);
    else
        hipLaunchKernelGGL(sample_rows<float>, dim3(blocks), dim3(SM_BLOCK), 0, st, a);
    return hipGetLastError();
}

}  // namespace osm
