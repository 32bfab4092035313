// Sampling a token of each row: temperature, top-k, top-p and min-p, with the
// random number given.
//
// With m the row's maximum, the weights are w_j = 2^{(x_j - m) log2(e) / T}.  Each
// filter keeps a prefix of the order "x descending, index ascending", so all
// of them together are one cut in that order:
//   top-k  the k-th element;
//   top-p  the first element at which the sum of weights, in that order and over
//          what top-k kept, reaches p times the whole;
//   min-p  the last element with w_j >= min_p (a test on the weight).
// The token is the first kept one, in index order, at which the running sum
// passes u times the sum of the kept weights.
//
// Nothing is sorted.  A row (or a chunk of it) is held in registers.  One pass adds
// every element to a histogram over w, 1/SUB of a power of two a bin, with
// the bin's weights (and for top-k their number); its running sums say in
// which bin a cut falls, and only that bin's elements are looked at one by one:
// ranked among each other if they are few, else by further histograms over
// their ordered bits and, among equal ones, their indices.  (bfloat16 rows of more than two
// vectors a lane of a workgroup go by their values instead: sample_values.hpp.)
//
// A binary64 weight is 20 instructions and a bin 10 more.  256 x 128256 binary32 without
// filters takes 47 to 50 us (the 131 MB at a large read's rate 19): 38 of them, timed without
// the ends of the rows, are the chunks, and the rest is what the ends add.  Few rows are
// bound by the end: 33 x 50257 binary32 with top-p and min-p 38 us, the chunks 8 of them;
// 1 x 32000 bfloat16 with top-k and top-p 18 and 5.  Short rows (4000 x 1000 binary32 top-k
// 28 to 29 us, the 16 MB 2.3) are bound by the wavefront's own steps, 2640 vector
// instructions a row.
//
// Weights are binary64 and the sums of a histogram are in fixed point: in
// binary32 the sums of 10^5 weights are off by more than the distance between the
// borders they put on [0, 1), and the token would depend on the order of the
// additions; integer sums do not depend on it.
#pragma once

#include "wide.hpp"
#include "kernels.h"

namespace osm {

// A row's team: W wavefronts (one, or the workgroup).
template <int W>
__device__ __forceinline__ void team_sync() {
    if constexpr (W == 1) wave_sync();
    else __syncthreads();
}

template <int W>
struct SampleShape {
    static constexpr int THREADS = 64 * W;
    // bins: 64 powers of two below the anchor, finer where rows are longer
    static constexpr int LOG_BINS = W == 1 ? 8 : 10;
    static constexpr int BINS = 1 << LOG_BINS;
    static constexpr int SUB = BINS / 64;
    static constexpr int PER = BINS / THREADS;  // bins a thread scans
    // elements of a cut's bin that are held
    static constexpr int CAP = W == 1 ? 512 : 3840;
};

template <int W>
struct SampleSmem {
    static constexpr int BINS = SampleShape<W>::BINS;
    union {
        uint64_t mass[BINS];   // a histogram of weights, in units of 2^-48
        double sums[BINS];     // the same, as numbers
    };
    union {
        uint32_t counts[BINS];  // a histogram of numbers, read before a cut's
        uint64_t bins[BINS];    // own histograms
        double seg[BINS];
    };
    uint64_t wave64[W];
    double waved[W];
    float wavef[W];
    uint32_t wave32[W];
    // (split rows) kept weights of each chunk: of the list, and of the bins kept whole
    uint64_t chunk[W > 1 ? 64 : 1];
    double whole[W > 1 ? 64 : 1];
    int found, n;
    uint64_t above, here;
    double base;
};

template <int W>
struct ListSmem : SampleSmem<W> {
    float lx[SampleShape<W>::CAP];  // the cut's bin: values and indices
    uint32_t li[SampleShape<W>::CAP];
};

// What a row asks for.
struct Rule {
    bool greedy;
    double c;        // log2(e) / T
    int64_t k;       // elements that top-k keeps (0: all)
    double p, q, u;  // 1: no top-p; 0: no min-p
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
    r.p = !(p < 1.0f) ? 1.0 : p > 0.0f ? (double)p : 0.0;  // (NaN: off)
    r.q = q > 0.0f ? __builtin_fmin((double)q, 1.0) : 0.0;
    r.u = u > 0.0f ? __builtin_fmin((double)u, 1.0) : 0.0;
    return r;
}

// A cut in the order: elements above x, and those equal to it up to index i, stay.
struct Cut {
    float x;
    uint32_t i;
    __device__ __forceinline__ bool keeps(float v, uint32_t at) const {
        return v > x || (v == x && at <= i);
    }
};

__device__ __forceinline__ Cut no_cut() { return Cut{-__builtin_inff(), 0xFFFFFFFFu}; }

// A weight (at most 1) in units of 2^-48, to nearest: the low bits of w + 16.
__device__ __forceinline__ uint64_t fixed48(double w) {
    return __builtin_bit_cast(uint64_t, w + 16.0) - 0x4030000000000000ull;
}

// ------------------------------------------------------------------ histograms
// The bin at which the running sum over sm.bins reaches `target`: sm.found, with
// the sum before it (which starts at `above`) in sm.above and its own in sm.here.
// p >= 0: the target is the part p of the sum, at least 1; the target is returned.
template <int W>
__device__ __forceinline__ uint64_t find_bin(SampleSmem<W>& sm, uint64_t above, uint64_t target,
                                             double p) {
    constexpr int PER = SampleShape<W>::PER;
    const int tid = threadIdx.x % (64 * W), lane = tid & 63, wv = tid >> 6;
    uint64_t v[PER], sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        v[j] = sm.bins[PER * tid + j];
        sum += v[j];
    }
    const uint64_t incl = wave_scan(sum);
    uint64_t before = above, total = above;
    if constexpr (W == 1) {
        total += lane_value(incl, 63);
    } else {
        if (lane == 63) sm.wave64[wv] = incl;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < wv) before += sm.wave64[w];
            total += sm.wave64[w];
        }
    }
    if (p >= 0.0) {
        const double want = __builtin_ceil(p * (double)total);
        target = want >= 1.0 ? (uint64_t)want : 1;
        target = target < total ? target : total;
    }
    before += incl - sum;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (before < target && target <= before + v[j]) {
            sm.found = PER * tid + j;
            sm.above = before;
            sm.here = v[j];
        }
        before += v[j];
    }
    team_sync<W>();
    return target;
}

template <int W>
__device__ __forceinline__ int bin_shift(uint32_t range) {
    const int bits = 32 - __builtin_clz(range | 1u);
    return bits > SampleShape<W>::LOG_BINS ? bits - SampleShape<W>::LOG_BINS : 0;
}

template <int W>
__device__ __forceinline__ void clear_bins(SampleSmem<W>& sm) {
    const int tid = threadIdx.x % (64 * W);
#pragma unroll
    for (int j = 0; j < SampleShape<W>::PER; ++j) sm.bins[tid + j * 64 * W] = 0;
    team_sync<W>();
}

__device__ __forceinline__ void add_bin(uint64_t& bin, uint64_t v) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&bin), (unsigned long long)v);
}

// Elements by place: a whole row in memory, or the held elements of a bin.
template <typename T>
struct RowSource {
    const T* x;
    int64_t n;
    __device__ __forceinline__ float value(int64_t i) const { return load1(x + i); }
    __device__ __forceinline__ uint32_t index(int64_t i) const { return (uint32_t)i; }
    __device__ __forceinline__ uint32_t end() const { return (uint32_t)(n - 1); }
};

struct ListSource {
    const float* x;
    const uint32_t* i;
    int64_t n;
    uint32_t last;  // largest index that can occur
    __device__ __forceinline__ float value(int64_t j) const { return x[j]; }
    __device__ __forceinline__ uint32_t index(int64_t j) const { return i[j]; }
    __device__ __forceinline__ uint32_t end() const { return last; }
};

// The cut behind the first `target` elements (MASS: units of weight; p >= 0: the
// part p of all of them) among those of `src` that `cut` keeps and whose order
// is within [lo, hi], by histograms over their order, then over the indices
// of equal ones.  units(x): a weight in fixed point.
template <bool MASS, int W, typename Src, typename Units>
__device__ __forceinline__ Cut find_cut(SampleSmem<W>& sm, const Src& src, uint32_t lo,
                                        uint32_t hi, Cut cut, uint64_t target, double p,
                                        const Units& units) {
    const int tid = threadIdx.x % (64 * W);
    uint64_t above = 0;
    bool first = true;
    for (;;) {  // rounds over values
        const int shift = bin_shift<W>(hi - lo);
        clear_bins(sm);
        for (int64_t j = tid; j < src.n; j += 64 * W) {
            const float x = src.value(j);
            const uint32_t k = order_key(x);
            if (k < lo || k > hi || !cut.keeps(x, src.index(j))) continue;
            add_bin(sm.bins[(hi - k) >> shift], MASS ? units(x) : 1);
        }
        team_sync<W>();
        target = find_bin(sm, above, target, first ? p : -1.0);
        first = false;
        above = sm.above;
        hi -= (uint32_t)sm.found << shift;
        if (shift == 0) break;
        const uint32_t width = (1u << shift) - 1;
        lo = hi - lo > width ? hi - width : lo;
        team_sync<W>();
    }
    // the value is that of hi; how many of the elements that hold it are kept
    const float v = order_value(hi);
    const uint64_t w = MASS ? units(v) : 1;
    const uint64_t ties = sm.here / w, need = (target - above + w - 1) / w;
    team_sync<W>();
    if (need >= ties) return Cut{v, v == cut.x ? cut.i : 0xFFFFFFFFu};
    uint32_t ilo = 0, ihi = src.end();
    above = 0;
    for (;;) {  // rounds over the indices of the ties
        const int shift = bin_shift<W>(ihi - ilo);
        clear_bins(sm);
        for (int64_t j = tid; j < src.n; j += 64 * W) {
            const float x = src.value(j);
            const uint32_t i = src.index(j);
            if (x == v && i >= ilo && i <= ihi && cut.keeps(x, i))
                add_bin(sm.bins[(i - ilo) >> shift], 1);
        }
        team_sync<W>();
        find_bin(sm, above, need, -1.0);
        above = sm.above;
        ilo += (uint32_t)sm.found << shift;
        team_sync<W>();
        if (shift == 0) return Cut{v, ilo};
        const uint32_t width = (1u << shift) - 1;
        ihi = ihi - ilo > width ? ilo + width : ihi;
    }
}

template <int W>
__device__ __forceinline__ uint32_t team_minimum(SampleSmem<W>& sm, uint32_t v) {
    v = ~group_max<64>(~v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) sm.wave32[threadIdx.x >> 6] = v;
        __syncthreads();
        v = sm.wave32[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = sm.wave32[w] < v ? sm.wave32[w] : v;
        __syncthreads();
    }
    return v;
}

// ------------------------------------------------- a row too odd for the short way
// Any row, by passes over memory: rows too long to be split, temperatures so low
// that logits over T leave 2^30, binary32 (or short) rows with a cut in a bin that holds
// more elements than fit or below the histogram's 64 powers of two, and numbers u at the
// very ends of [0, 1] of split rows with a filter.  A long row takes several times as long
// (64 x 128256 binary32, a top-k of 50 at T 0.1: 450 us; at T 1 73).
template <int W, typename T>
__device__ __forceinline__ void sample_row(SampleSmem<W>& sm, const RowSource<T>& src,
                                           const Rule& r, float* val, int32_t* idx) {
    constexpr int BINS = SampleShape<W>::BINS, PER = SampleShape<W>::PER;
    const int tid = threadIdx.x % (64 * W), lane = tid & 63, wv = tid >> 6;
    // the maximum with its lowest index, the minimum, and whether a NaN or +inf is there
    uint64_t best = 0;
    uint32_t least = ~0u;
    int bad = 0;
    for (int64_t i = tid; i < src.n; i += 64 * W) {
        const float x = src.value(i);
        bad |= !(x < __builtin_inff());
        const uint64_t k = (uint64_t)order_key(x) << 32 | (uint32_t)~(uint32_t)i;
        best = k > best ? k : best;
        least = (uint32_t)(k >> 32) < least ? (uint32_t)(k >> 32) : least;
    }
    best = group_max<64>(best);
    bad = __any(bad);
    if constexpr (W > 1) {
        __syncthreads();
        if (lane == 0) {
            sm.wave64[wv] = best;
            sm.wave32[wv] = (uint32_t)bad;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) {
            best = sm.wave64[w] > best ? sm.wave64[w] : best;
            bad |= (int)sm.wave32[w];
        }
    }
    team_sync<W>();
    const float mx = order_value((uint32_t)(best >> 32));
    if (bad || mx == -__builtin_inff() || r.greedy) {
        if (tid == 0) {
            const bool none = bad || mx == -__builtin_inff();
            *idx = none ? -1 : (int32_t)~(uint32_t)best;
            *val = none ? __builtin_nanf("") : 1.0f;
        }
        return;
    }
    const double m = mx, c = r.c;
    const auto wt = [m, c](float x) { return exp2_wide(((double)x - m) * c); };
    const uint32_t top = (uint32_t)(best >> 32), bottom = team_minimum(sm, least);
    Cut cut = no_cut();
    // the largest weight, 1, in so many units that n of them sum below 2^63
    const double scale = __builtin_ldexp(1.0, 62 - (64 - __builtin_clzll((uint64_t)src.n)));
    const auto units = [&](float x) { return (uint64_t)__builtin_fma(wt(x), scale, 0.5); };
    if (r.k) cut = find_cut<false>(sm, src, bottom, top, cut, (uint64_t)r.k, -1.0, units);
    if (r.p < 1.0) cut = find_cut<true>(sm, src, bottom, top, cut, 0, r.p, units);

    // the token: sums of up to BINS segments of the range, then the segment that
    // the target falls into as the next range
    const double q = r.q;
    const auto kept = [&](int64_t i) {
        const float x = src.value(i);
        const double w = wt(x);
        return cut.keeps(x, (uint32_t)i) && w >= q ? w : 0.0;
    };
    int64_t a = 0, b = src.n;
    double target = 0.0, total = 0.0;
    bool first = true;
    do {
        int64_t L = (b - a + BINS - 1) / BINS;
        L = (L + 63) / 64 * 64;
        // (the segments past the range are empty)
        for (int s = tid; s < BINS; s += 64 * W)
            if (a + s * L >= b) sm.seg[s] = 0.0;
        for (int s = wv; s < BINS && a + s * L < b; s += W) {
            double sum = 0.0;
            const int64_t e = a + (s + 1) * L < b ? a + (s + 1) * L : b;
            for (int64_t i = a + s * L + lane; i < e; i += 64) sum += kept(i);
            sum = group_sum<64>(sum);
            if (lane == 0) sm.seg[s] = sum;
        }
        if (tid == 0) sm.found = BINS;
        team_sync<W>();
        double s[PER], sum = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            s[j] = sm.seg[PER * tid + j];
            sum += s[j];
        }
        const double incl = wave_scan(sum);
        double before = lane_before(incl), all = lane_value(incl, 63);
        if constexpr (W > 1) {
            if (lane == 63) sm.waved[wv] = incl;
            __syncthreads();
            double o = 0.0;
            all = 0.0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (w < wv) o += sm.waved[w];
                all += sm.waved[w];
            }
            before += o;
        }
        if (first) {
            total = all;
            target = r.u * all;
            first = false;
        }
        double start[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            start[j] = before;
            before += s[j];
            if (s[j] > 0.0 && before > target) atomicMin(&sm.found, PER * tid + j);
        }
        team_sync<W>();
        int at = sm.found;
        team_sync<W>();
        if (at == BINS) {  // a rounding left the target unreached: the last of any weight
            if (tid == 0) sm.found = -1;
            team_sync<W>();
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (s[j] > 0.0) atomicMax(&sm.found, PER * tid + j);
            team_sync<W>();
            at = sm.found;
            target = __builtin_inf();
        }
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (PER * tid + j == at) sm.base = start[j];
        team_sync<W>();
        target -= sm.base;
        a += at * L;
        b = a + L < b ? a + L : b;
        team_sync<W>();
    } while (b - a > 64);
    if (wv == 0) {
        const int64_t i = a + lane;
        const double w = i < b ? kept(i) : 0.0;
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

// --------------------------------------------------------- rows held in registers
__device__ __forceinline__ float elem(const u32x4& q, int e, float*) {
    return __uint_as_float(q[e]);
}
__device__ __forceinline__ float elem(const u32x4& q, int e, bf16_t*) {
    return e & 1 ? bf16_hi(q[e >> 1]) : bf16_lo(q[e >> 1]);
}

// L elements at x by a team: 16-byte vector r * THREADS + thread in q[r], counted from
// the 16-byte line that x lies in.  What lies before x or past its end reads as
// -inf, an element that no filter keeps; nothing outside is loaded.
template <typename T, int W, int R>
struct Held {
    static constexpr int E = Vec<T>::N;
    static constexpr int64_t ELEMS = (int64_t)64 * W * R * E;  // (E - 1 fewer where x is unaligned)
    u32x4 q[R];
    int32_t first;  // index of q[0]'s first element, from x

    __device__ __forceinline__ void load(const T* x, int32_t L) {
        const int tid = threadIdx.x % (64 * W);
        const int h = (int)(((uintptr_t)x & 15) / sizeof(T));
        first = tid * E - h;
        constexpr uint32_t PAD = E == 4 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int32_t i = first + r * 64 * W * E;
            if (i >= 0 && i + E <= L) {
                q[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + i));
            } else {
                q[r] = u32x4{PAD, PAD, PAD, PAD};
                if (i < L && i + E > 0) {  // the two ends
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (i + e < 0 || i + e >= L) continue;
                        if constexpr (E == 4) {
                            q[r][e] = __float_as_uint(x[i + e]);
                        } else {
                            const uint32_t b = x[i + e].bits;
                            q[r][e >> 1] = e & 1 ? (q[r][e >> 1] & 0xFFFFu) | b << 16
                                                 : (q[r][e >> 1] & 0xFFFF0000u) | b;
                        }
                    }
                }
            }
        }
    }
    // f(vector, index of its first element) for each, in a loop over registers that turn.
    // Unrolled, the kernel's code is several times the instruction cache (211 KB), and the
    // end of a row, which each CU runs a few times, waits for its code
    template <typename F>
    __device__ __forceinline__ void each(const F& f) {
        constexpr int STEP = R % 2 == 0 && E == 4 ? 2 : 1;
#pragma unroll 1
        for (int r = 0; r < R; r += STEP) {
            u32x4 head[STEP];
#pragma unroll
            for (int s = 0; s < STEP; ++s) {
                head[s] = q[s];
                f(q[s], first + (r + s) * 64 * W * E);
            }
#pragma unroll
            for (int j = 0; j + STEP < R; ++j) q[j] = q[j + STEP];
#pragma unroll
            for (int s = 0; s < STEP; ++s) q[R - STEP + s] = head[s];
        }
    }
    // the registers turn by one vector
    __device__ __forceinline__ void turn() {
        const u32x4 head = q[0];
#pragma unroll
        for (int j = 0; j + 1 < R; ++j) q[j] = q[j + 1];
        q[R - 1] = head;
    }
    __device__ __forceinline__ static float at(const u32x4& v, int e) {
        return elem(v, e, (T*)nullptr);
    }
    // (NaN where there is one)
    __device__ __forceinline__ float maximum() const {
        float m = -__builtin_inff();
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < E; e += 2)
                m = __builtin_elementwise_maximum(
                    __builtin_elementwise_maximum(at(q[r], e), at(q[r], e + 1)), m);
        return m;
    }
};

template <int STEP = 0>
__device__ __forceinline__ float wave_maximum(float v) {
    if constexpr (STEP < 6) {
        float a, b;
        bfly_operands<STEP>(v, a, b);
        return wave_maximum<STEP + 1>(__builtin_elementwise_maximum(a, b));
    } else {
        return v;
    }
}

template <int W>
__device__ __forceinline__ float team_maximum(SampleSmem<W>& sm, float v) {
    v = wave_maximum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) sm.wavef[threadIdx.x >> 6] = v;
        __syncthreads();
        v = sm.wavef[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = __builtin_elementwise_maximum(v, sm.wavef[w]);
        __syncthreads();
    }
    return v;
}

template <int W>
__device__ __forceinline__ double team_sum(SampleSmem<W>& sm, double v) {
    v = group_sum<64>(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) sm.waved[threadIdx.x >> 6] = v;
        __syncthreads();
        v = sm.waved[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += sm.waved[w];
        __syncthreads();
    }
    return v;
}

// Weights 2^t relative to the maximum m of a row or a chunk, which is exactly 1, and
// their bins in a histogram, 1/SUB of a power of two a bin.  Bins are counted down from
// a power of two, 2^0 standing for the value a / c just above m, so that the bins
// of another chunk are the same ones but for a shift by the difference of their a.
// (m c has to be small enough for its ceiling to be one.)
struct Anchor {
    double m, c, a, shift;  // shift: of the maximum, in (-1, 0]
    Exp2 exp2;
    // (weights vanish below 2^-1075; the bound also takes the place of -inf and NaN)
    __device__ __forceinline__ double t(float x) const {
        return __builtin_fmax(((double)x - m) * c, -1100.0);
    }
    __device__ __forceinline__ double weight(float x) const { return exp2(t(x)); }
    // the low bits of s + 1.5 2^52 / SUB are round(s SUB)
    template <int W>
    __device__ __forceinline__ int bin(double t) const {
        constexpr double M = 0x1.8p52 / SampleShape<W>::SUB;
        return -(int)(uint32_t)__builtin_bit_cast(uint64_t, t + shift + M);
    }
};

constexpr double kAnchorMax = 0x1p30;
__device__ __forceinline__ bool cold(double mc) { return !(__builtin_fabs(mc) <= kAnchorMax); }
__device__ __forceinline__ Anchor anchor(float m, double c) {
    const double mc = (double)m * c, a = __builtin_ceil(mc);
    return Anchor{(double)m, c, a, mc - a, Exp2::make()};
}

// Adds the held elements to the histogram sm.mass of weights (MASS) and to that of
// their numbers sm.counts (COUNT).  The last bin stands for everything below the
// window and stays empty; returns whether an element there has a weight at all.
template <bool MASS, bool COUNT, typename T, int W, int R>
__device__ __forceinline__ bool add_histogram(SampleSmem<W>& sm, Held<T, W, R>& h,
                                              const Anchor& an) {
    bool tail = false;
    h.each([&](const u32x4& v, int32_t) {
#pragma unroll
        for (int e = 0; e < h.E; ++e) {
            const double t = an.t(h.at(v, e));
            const int b = an.bin<W>(t);
            const uint64_t w = MASS ? fixed48(an.exp2(t)) : 0;
            if (b < SampleShape<W>::BINS - 1) {
                if constexpr (MASS) add_bin(sm.mass[b], w);
                if constexpr (COUNT) atomicAdd(&sm.counts[b], 1u);
            }
            if constexpr (COUNT) tail |= b >= SampleShape<W>::BINS - 1 && t > -1080.0;
        }
    });
    return tail;
}

// The sum of the held elements' weights.
template <typename T, int W, int R>
__device__ __forceinline__ double sum_weights(SampleSmem<W>& sm, Held<T, W, R>& h,
                                              const Anchor& an) {
    double z = 0.0;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < h.E; ++e) z += an.weight(h.at(h.q[r], e));
    return team_sum(sm, z);
}

// The lowest index of a held element equal to m.
template <typename T, int W, int R>
__device__ __forceinline__ uint32_t index_of(SampleSmem<W>& sm, Held<T, W, R>& h, float m) {
    uint32_t at = ~0u;
    h.each([&](const u32x4& v, int32_t i) {
#pragma unroll
        for (int e = 0; e < h.E; ++e)
            at = h.at(v, e) == m && (uint32_t)(i + e) < at ? (uint32_t)(i + e) : at;
    });
    return team_minimum(sm, at);
}

// Values that a range of bins can hold, and a bit more.
struct Range {
    int lo, hi;   // bins
    float x0, x1;
    template <int W>
    __device__ __forceinline__ static Range of(int lo, int hi, const Anchor& an) {
        Range g{lo, hi, -__builtin_inff(), __builtin_inff()};
        const double half = 0.5 / SampleShape<W>::SUB, near = 1e-9 * __builtin_fabs(an.m);
        const double e0 = (an.a - (hi / (double)SampleShape<W>::SUB + half)) / an.c;
        const double e1 = (an.a - (lo / (double)SampleShape<W>::SUB - half)) / an.c;
        if (an.c > 0.0) {
            g.x0 = (float)(e0 - 1e-6 * __builtin_fabs(e0) - near);
            g.x1 = lo > 0 ? (float)(e1 + 1e-6 * __builtin_fabs(e1) + near) : g.x1;
        }
        return g;
    }
};

// Whether x may be in the range.
__device__ __forceinline__ bool near(const Range& g, float x) { return x >= g.x0 && x <= g.x1; }

// Appends x to the list if its bin is in the range; all lanes call.
template <int W>
__device__ __forceinline__ void append(ListSmem<W>& sm, const Range& g, const Anchor& an,
                                       float x, uint32_t i) {
    bool in = near(g, x);
    if (__ballot(in) == 0) return;
    const int b = an.bin<W>(an.t(x));
    in = in && b >= g.lo && b <= g.hi;
    const uint64_t who = __ballot(in);
    if (who == 0) return;
    const int lane = threadIdx.x & 63;
    int at = 0;
    if (lane == 0) at = atomicAdd(&sm.n, __popcll(who));
    at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((1ull << lane) - 1));
    if (in && at < SampleShape<W>::CAP) {
        sm.lx[at] = x;
        sm.li[at] = i;
    }
}

// The cut behind the first `target` units (MASS: of weight, else elements) of the list's
// kept elements, 1 <= target <= their sum.
template <bool MASS, int W>
__device__ __forceinline__ Cut list_cut(ListSmem<W>& sm, int n, Cut cut, uint64_t target,
                                        const Anchor& an, uint32_t last) {
    const auto units = [an](float x) { return fixed48(an.weight(x)); };
    if (n > 64) {
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        for (int j = threadIdx.x % (64 * W); j < n; j += 64 * W) {
            const uint32_t k = order_key(sm.lx[j]);
            lo = k < lo ? k : lo;
            hi = k > hi ? k : hi;
        }
        lo = team_minimum(sm, lo);
        hi = ~team_minimum(sm, ~hi);
        const ListSource src{sm.lx, sm.li, n, last};
        return find_cut<MASS>(sm, src, lo, hi, cut, target, -1.0, units);
    }
    // an element a lane: the units of those at or before it in the order
    if (threadIdx.x % (64 * W) < 64) {
        const int lane = threadIdx.x & 63;
        const float x = lane < n ? sm.lx[lane] : 0.0f;
        const uint32_t i = lane < n ? sm.li[lane] : 0u;
        const bool in = lane < n && cut.keeps(x, i);
        const uint64_t w = !in ? 0 : MASS ? units(x) : 1;
        uint64_t incl = 0;
        for (int l = 0; l < n; ++l) {
            const float xl = lane_value(x, l);
            const uint32_t il = lane_value(i, l);
            const uint64_t wl = lane_value(w, l);
            incl += xl > x || (xl == x && il <= i) ? wl : 0;
        }
        if (in && incl >= target && incl - w < target) {
            sm.base = (double)x;
            sm.found = (int)i;
        }
    }
    team_sync<W>();
    const Cut c{(float)sm.base, (uint32_t)sm.found};
    team_sync<W>();
    return c;
}

template <int STEP = 0>
__device__ __forceinline__ uint64_t wave_total(uint64_t v) {
    if constexpr (STEP < 6) {
        uint64_t a, b;
        bfly_operands64<STEP>(v, a, b);
        return wave_total<STEP + 1>(a + b);
    } else {
        return v;
    }
}

// Sum of the list's kept weights, in units.
template <int W>
__device__ __forceinline__ uint64_t list_sum(ListSmem<W>& sm, int n, Cut cut,
                                             const Anchor& an) {
    uint64_t s = 0;
    for (int j = threadIdx.x % (64 * W); j < n; j += 64 * W)
        if (cut.keeps(sm.lx[j], sm.li[j])) s += fixed48(an.weight(sm.lx[j]));
    s = wave_total(s);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) sm.wave64[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) s += sm.wave64[w];
        __syncthreads();
    }
    return s;
}

// The first bin below `limit` at which the running sum of sm.sums reaches p times (their
// sum + extra), the sum before it in sm.base; BINS if none does.  all: their sum.
template <int W>
__device__ __forceinline__ int find_mass(SampleSmem<W>& sm, int limit, double extra, double p,
                                         double* all, double* need) {
    constexpr int PER = SampleShape<W>::PER, BINS = SampleShape<W>::BINS;
    const int tid = threadIdx.x % (64 * W), lane = tid & 63, wv = tid >> 6;
    double v[PER], sum = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        v[j] = PER * tid + j < limit ? sm.sums[PER * tid + j] : 0.0;
        sum += v[j];
    }
    const double incl = wave_scan(sum);
    double before = lane_before(incl), total = lane_value(incl, 63);
    if (tid == 0) sm.found = BINS;
    if constexpr (W > 1) {
        if (lane == 63) sm.waved[wv] = incl;
        __syncthreads();
        double o = 0.0;
        total = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < wv) o += sm.waved[w];
            total += sm.waved[w];
        }
        before += o;
    } else {
        wave_sync();
    }
    const double target = p * (total + extra);
    double start[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        start[j] = before;
        before += v[j];
        if (v[j] > 0.0 && before >= target) atomicMin(&sm.found, PER * tid + j);
    }
    team_sync<W>();
    const int at = sm.found;
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (PER * tid + j == at) sm.base = start[j];
    team_sync<W>();
    *all = total;
    *need = target - (at < BINS ? sm.base : total);
    team_sync<W>();
    return at;
}

// The first bin at which the running sum of sm.counts reaches k, the sum before it in
// *above; BINS if none does.
template <int W>
__device__ __forceinline__ int find_count(SampleSmem<W>& sm, int64_t k, uint64_t* above,
                                          uint64_t* here) {
    constexpr int PER = SampleShape<W>::PER, BINS = SampleShape<W>::BINS;
    const int tid = threadIdx.x % (64 * W), lane = tid & 63, wv = tid >> 6;
    uint32_t v[PER], sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        v[j] = sm.counts[PER * tid + j];
        sum += v[j];
    }
    const uint32_t incl = wave_scan(sum);
    uint32_t before = incl - sum;
    if (tid == 0) sm.found = BINS;
    if constexpr (W > 1) {
        if (lane == 63) sm.wave32[wv] = incl;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < wv) before += sm.wave32[w];
    } else {
        wave_sync();
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if ((int64_t)before < k && k <= (int64_t)before + v[j]) {
            sm.found = PER * tid + j;
            sm.above = before;
            sm.here = v[j];
        }
        before += v[j];
    }
    team_sync<W>();
    const int at = sm.found;
    *above = sm.above;
    *here = sm.here;
    team_sync<W>();
    return at;
}

// What the filters leave of a row whose histogram is complete (weights in sm.sums,
// numbers in sm.counts for a top-k; both relative to `an`): a cut, and the bins of
// which it says all: those below `sure` are kept whole, those above `last` dropped whole.
struct Filtered {
    Cut cut;
    int sure, last;
    bool ok;  // false: the histogram does not decide
};

// gather(range) appends the row's elements in a range of bins to the list.
// sums: whether the caller wants the list to hold every element whose bin is neither
// kept nor dropped whole.
template <int W, typename Gather>
__device__ __forceinline__ Filtered filter_row(ListSmem<W>& sm, const Rule& r, const Anchor& an,
                                               bool tail, uint32_t last_index, bool sums,
                                               const Gather& gather) {
    constexpr int BINS = SampleShape<W>::BINS, CAP = SampleShape<W>::CAP;
    const int tid = threadIdx.x % (64 * W);
    Filtered f{no_cut(), BINS - 1, BINS - 1, true};
    int held0 = 0, held1 = -1, n = 0;  // bins whose elements are in the list
    double extra = 0.0;
    int limit = BINS - 1;
    const double log_q = r.q > 0.0 ? (double)__builtin_log2f((float)r.q) : -1100.0;
    // one after the other: top-k, top-p, min-p; each wants the elements of some bins
#pragma unroll 1
    for (int step = 0; step < 3; ++step) {
        int lo = 0, hi = -1;
        uint64_t above = 0, here = 0;
        double need = 0.0;
        if (step == 0) {
            if (!r.k) continue;
            const int b = find_count(sm, r.k, &above, &here);
            if (b == BINS) {
                if (!tail) continue;  // fewer elements than k have any weight
                f.ok = false;         // the k-th is below the window
                return f;
            }
            // (with the elements above it, if they all fit)
            lo = above + here <= (uint64_t)CAP ? 0 : b;
            hi = b;
            if (lo == 0) {
                here += above;
                above = 0;
            }
        } else if (step == 1) {
            if (!(r.p < 1.0)) continue;
            double all;
            const int b = find_mass(sm, limit, extra, r.p, &all, &need);
            // (min-p alone cuts where its bin is clearly before this one)
            if (b < BINS && an.bin<W>(log_q) + 1 < b) continue;
            if (b < BINS) lo = hi = b;
            else if (limit == BINS - 1) continue;  // (a rounding: nothing to cut off)
        } else {
            if (!sums) break;
            if (r.q > 0.0) {  // w >= q, somewhere in the bins around that
                const int b = an.bin<W>(log_q);
                f.sure = b - 1 < f.sure ? (b > 1 ? b - 1 : 0) : f.sure;
                f.last = b + 1 < f.last ? b + 1 : f.last;
                f.sure = f.sure < f.last ? f.sure : f.last;
            }
            if (f.sure == BINS - 1 || (held0 <= f.sure && f.last <= held1)) break;
            lo = f.sure;
            hi = f.last;
        }
        if (lo <= hi) {
            if (tid == 0) sm.n = 0;
            team_sync<W>();
            gather(Range::of<W>(lo, hi, an));
            team_sync<W>();
            n = sm.n;
            held0 = lo;
            held1 = hi;
            // (a rounding can take an element out of its bin)
            if (n > CAP || (step == 0 && (uint64_t)n != here)) f.ok = false;
            team_sync<W>();
            if (!f.ok) return f;
        }
        if (step == 0) {
            f.cut = list_cut<false>(sm, n, f.cut, (uint64_t)r.k - above, an, last_index);
            limit = lo;
            if (r.p < 1.0) extra = (double)list_sum(sm, n, f.cut, an) * 0x1p-48;
        } else if (step == 1) {
            const uint64_t total = list_sum(sm, n, f.cut, an);
            const double want = __builtin_ceil(need * 0x1p48);
            uint64_t target = want >= 1.0 ? (uint64_t)want : 1;
            target = target < total ? target : total;
            if (target == 0) {
                f.ok = false;
                return f;
            }
            f.cut = list_cut<true>(sm, n, f.cut, target, an, last_index);
        }
        if (step < 2 && lo <= hi) {
            f.sure = lo;
            f.last = hi;
        }
    }
    return f;
}

// The token of a row of which `h` holds all, or the part that the target falls into:
// the first element, in index order, at which the running sum of the weights that
// wt(vector, index of its first element, weights) gives passes the target u * sum (PART:
// what is left of it, of a row whose sum is `total`).  base: added to the index.  False
// if no element has a weight.
template <bool PART, typename T, int W, int R, typename Wt>
__device__ __forceinline__ bool locate(SampleSmem<W>& sm, Held<T, W, R>& h, const Wt& wt,
                                       double target, double total, uint32_t base, float* val,
                                       int32_t* idx) {
    static_assert(R * W <= 64, "a lane a segment");
    const int lane = threadIdx.x & 63, wv = (threadIdx.x % (64 * W)) >> 6;
    // segments of 64 vectors, in index order: their sums, then (the last turn) the weights
    // in the one that the target falls into, by the wavefront that has it
    u32x4 q = h.q[0];
    uint32_t i0 = (uint32_t)h.first;
    constexpr int E = Held<T, W, R>::E;
    double w[E], v, found_sum = 0.0;
    bool reached = false;
    int turn = 0;
#pragma unroll 1
    for (;; ++turn) {
        wt(q, i0, w);
        v = 0.0;
#pragma unroll
        for (int e = 0; e < h.E; ++e) v += w[e];
        if (turn == R) break;
        const double s = group_sum<64>(v);
        if (lane == 0) sm.seg[turn * W + wv] = s;
        h.turn();
        q = h.q[0];
        i0 += 64 * W * h.E;
        if (turn + 1 < R) continue;
        team_sync<W>();
        const double seg = lane < R * W ? sm.seg[lane] : 0.0;
        const double incl = wave_scan(seg);
        if constexpr (!PART) {
            total = lane_value(incl, 63);
            target *= total;
        }
        const uint64_t some = __ballot(seg > 0.0);
        if (some == 0) return false;
        // (the last of any weight stands in where a rounding leaves the target unreached)
        const uint64_t past = __ballot(seg > 0.0 && incl > target);
        const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
        if (at % W != wv) return true;
        reached = past != 0;
        found_sum = at ? lane_value(incl, at - 1) : 0.0;
        for (int r = 0; r < at / W; ++r) h.turn();
        q = h.q[0];
        for (int r = at / W; r < R; ++r) h.turn();
        i0 = (uint32_t)(h.first + at / W * 64 * W * h.E);
    }
    target = reached ? target - found_sum : __builtin_inf();
    const double run = wave_scan(v);
    const double prev = lane_before(run);
    const uint64_t mine = __ballot(v > 0.0), over = __ballot(v > 0.0 && run > target);
    const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(mine);
    if (lane == l) {
        const double rest = over ? target - prev : __builtin_inf();
        double sum = 0.0, w1 = 0.0;
        uint32_t i1 = 0;
        bool done = false;
#pragma unroll
        for (int e = 0; e < h.E; ++e) {
            sum += w[e];
            if (w[e] > 0.0 && !done) {
                i1 = i0 + e;
                w1 = w[e];
                done = sum > rest;
            }
        }
        *idx = (int32_t)(base + i1);
        *val = (float)(w1 / total);
    }
    return true;
}

}  // namespace osm
