// Sampling of bfloat16 rows by the values themselves.  Between 2^-11 and 2^5 there are
// only 2 x 2048 of them, so the histogram has a bin for each and counts: no weight is
// computed per element, every bin is exact, and the cuts (sample.hpp) follow from the
// bins alone, to the number of equal elements that stay.  The few elements nearer to 0,
// which in the order stand between the positive and the negative bins, and those
// beyond the negative end are weighed one by one, as two classes, which are looked at again
// only if a cut falls inside.  Rows with larger values, or none near 0, move the 16
// octaves up, and parts of a row that moved them elsewhere are brought into line at
// its end (64 x 128256 with 20 added to all, where a row's parts have their maxima on both
// sides of 2^5: 40 us; centred 38).
//
// Against a histogram of weights this takes a third of the instructions an element and no
// second pass over the row: 512 x 128256 top-p 204 -> 146 us when it came, 64 x 128256 with a
// setting a row 91 -> 60; now 100 and 35.  What bounds it is not the 131 MB (19 us at a large
// read's rate): the chunks take 57 of the 100 us, with 1000 vector instructions and 53
// shared-memory ones a wavefront, ends included, and the ends of the rows the rest.
#pragma once

#include "sample.hpp"

namespace osm {

constexpr int VB_SIDE = 2048;           // bins of a sign: 16 octaves
constexpr int VB_BINS = 2 * VB_SIDE;
constexpr int VB_PER = VB_BINS / 512;   // bins a thread, in the order of the values
static_assert(VB_PER == 8, "eight bins are one 16-byte load of a chunk's counts");
static_assert(VB_SIDE * 4 == 1 << 13, "the sign's place in a byte address");

struct ValueSmem {
    SampleSmem<8> s;
    // of a pattern: sign * 2048 + (magnitude - base); for those outside one a lane, so
    // that a masked row's additions do not wait for each other
    uint32_t values[VB_BINS + 64];
    union {
        double weights[VB_BINS];  // what an element of a bin weighs, if it is kept
        struct {                  // before that: the elements of a class in which a cut falls
            float lx[VB_BINS];
            uint32_t li[VB_BINS];
        };
    };
    uint64_t mid, tail;        // weights of the classes, in units of 2^-48
    uint32_t mid_n, tail_n;
    double part[8][64];        // kept weights by wavefront and chunk
    uint32_t take[64];         // of the cut's value: elements kept of each chunk,
    uint32_t have[64];         // and elements there
    float val;
    int32_t idx;
};


// Magnitude (the pattern without its sign) of the first bins: 15 octaves below the octave
// of m, or of 2^4 if that is larger; for m up to -8 the octave of m itself, since all
// elements are at least as far from 0.  Both in steps of four octaves, so that the bins of
// a row's chunks are the same ones but for a shift of whole 512.  A chunk whose bins
// begin below the row's has a smaller maximum, or none above 0; one whose bins begin above
// the row's has only negative elements, and none nearer to 0 than its bins.
__device__ __forceinline__ int value_base(float m) {
    const int e = (int)(__float_as_uint(m) >> 23 & 0xFF);
    const int up = m > -8.0f ? (m < 0.0f ? 0 : (e - 128) / 4) : (e - 116) / 4;
    const int first = 116 + 4 * (up > 0 ? up : 0);
    return (first < 240 ? first : 240) << 7;
}

// The value of a bin in the order: positions 0 .. 2047 are the positive ones, largest
// first, the others the negative ones.
__device__ __forceinline__ float position_value(int p, int base) {
    const uint32_t mag = (uint32_t)(base + (p < VB_SIDE ? VB_SIDE - 1 - p : p - VB_SIDE));
    return __uint_as_float((p < VB_SIDE ? 0u : 0x80000000u) | mag << 16);
}

__device__ __forceinline__ void clear_values(ValueSmem& sm) {
#pragma unroll
    for (int j = 0; j < VB_PER; ++j) sm.values[threadIdx.x + j * 512] = 0;
    if (threadIdx.x == 0) {
        sm.mid = sm.tail = 0;
        sm.mid_n = sm.tail_n = 0;
    }
}

// The bin of a pattern, VB_BINS outside of them.
__device__ __forceinline__ uint32_t value_bin(uint32_t bits, uint32_t base) {
    const uint32_t rel = (bits & 0x7FFFu) - base;
    return rel < (uint32_t)VB_SIDE ? (bits >> 4 & (uint32_t)VB_SIDE) | rel : (uint32_t)VB_BINS;
}

__device__ __forceinline__ uint32_t pattern(const u32x4& v, int e) {
    return e & 1 ? v[e >> 1] >> 16 : v[e >> 1] & 0xFFFFu;
}

// Adds the held elements.  Those whose weight vanishes count nowhere.
template <int R>
__device__ __forceinline__ void add_values(ValueSmem& sm, Held<bf16_t, 8, R>& h, const Anchor& an) {
    const uint32_t base = (uint32_t)value_base((float)an.m);
    // patterns of negative elements whose weight is below 2^-1100 (-inf: always)
    const float zero = (float)(an.m - 1100.0 / an.c);
    const uint32_t gone = 0x8000u + (!(an.c > 0.0)  ? 0x7F80u
                                     : zero < 0.0f ? (__float_as_uint(-zero) >> 16) + 1
                                                   : 0u);
    const uint32_t outside = 4u * (VB_BINS + (threadIdx.x & 63));
    h.each([&](const u32x4& v, int32_t) {
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // four times the bin: a byte address
            const uint32_t word = v[e >> 1], mag = e & 1 ? word >> 16 & 0x7FFFu : word & 0x7FFFu;
            const uint32_t sign = e & 1 ? word >> 31 : word >> 15 & 1u;
            const uint32_t rel = (mag << 2) - (base << 2);
            const bool out = rel >= 4u * VB_SIDE;
            const uint32_t at = out ? outside : sign << 13 | rel;
            atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(sm.values) + at), 1u);
            odd |= out;
        }
        if (!__any(odd)) return;
        uint32_t which = 0;  // the lane's elements of a class
#pragma unroll
        for (int e = 0; e < 8; ++e)
            which |= value_bin(pattern(v, e), base) == (uint32_t)VB_BINS && pattern(v, e) < gone
                         ? 1u << e
                         : 0u;
        while (__any(which != 0)) {
            const int e = which ? __builtin_ctz(which) : 0;
            const uint32_t word = e < 2 ? v[0] : e < 4 ? v[1] : e < 6 ? v[2] : v[3];
            const uint32_t bits = e & 1 ? word >> 16 : word & 0xFFFFu;
            const double t = an.t(__uint_as_float(bits << 16));
            if (which && t > -1080.0) {
                const uint64_t w = fixed48(an.exp2(t));
                const bool middle = (bits & 0x7FFFu) < base;
                add_bin(middle ? sm.mid : sm.tail, w);
                atomicAdd(middle ? &sm.mid_n : &sm.tail_n, 1u);
            }
            which &= which - 1;
        }
    });
}

// What a chunk's classes leave.
struct ClassSum {
    uint64_t mid, tail;   // units of 2^-48 of the chunk's maximum
    uint32_t mid_n, tail_n;
};

// A thread's bins, one after the other in a loop: f(number, weight, position).  The
// registers turn (see Held::each): the end of a row runs once in a while, and what
// bounds it is the fetching of its code, not its work.
struct Bins {
    uint32_t n[VB_PER];
    double w[VB_PER];
    template <typename F>
    __device__ __forceinline__ void each(const F& f) {
        int p = VB_PER * (int)threadIdx.x;
#pragma unroll 1
        for (int j = 0; j < VB_PER; ++j, ++p) {
            f(n[0], w[0], p);
            const uint32_t n0 = n[0];
            const double w0 = w[0];
#pragma unroll
            for (int i = 0; i + 1 < VB_PER; ++i) {
                n[i] = n[i + 1];
                w[i] = w[i + 1];
            }
            n[VB_PER - 1] = n0;
            w[VB_PER - 1] = w0;
        }
    }
};

// The classes of chunk `lane` in the row's terms; part: what the chunk's maximum weighs there.
struct Classes {
    double mid, tail;
    uint32_t mid_n, tail_n;
};
__device__ __forceinline__ Classes in_row(const ClassSum& c, double part) {
    return Classes{(double)c.mid * 0x1p-48 * part, (double)c.tail * 0x1p-48 * part,
                   part > 0.0 ? c.mid_n : 0u, part > 0.0 ? c.tail_n : 0u};
}

// Words that workgroups leave for each other, at the device's coherence point.
__device__ __forceinline__ void put(uint64_t* p, uint64_t v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put(uint32_t* p, uint32_t v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get(const uint64_t* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t get(const uint32_t* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The numbers of chunk c at positions p .. p + 7, 16 bits each, in the order of the patterns'
// bins (from the last for positive values): in the scratch of a split row, or the bins of
// a held one.
struct ScratchCounts {
    uint64_t* words;
    __device__ __forceinline__ uint64_t* at(int c, int p) const {
        return words + (int64_t)c * (VB_BINS / 4) +
               (p < VB_SIDE ? VB_SIDE - VB_PER - p : p) / 4;
    }
    __device__ __forceinline__ void operator()(int c, int p, uint64_t (&q)[2]) const {
        q[0] = get(at(c, p));
        q[1] = get(at(c, p) + 1);
    }
    __device__ __forceinline__ void replace(int c, int p, const uint64_t (&q)[2]) const {
        put(at(c, p), q[0]);
        put(at(c, p) + 1, q[1]);
    }
};
struct HeldCounts {
    const uint32_t* values;
    __device__ __forceinline__ void operator()(int, int p, uint64_t (&q)[2]) const {
        const uint32_t* v = values + (p < VB_SIDE ? VB_SIDE - VB_PER - p : p);
        q[0] = (uint64_t)(v[2] | v[3] << 16) << 32 | (v[0] | v[1] << 16);
        q[1] = (uint64_t)(v[6] | v[7] << 16) << 32 | (v[4] | v[5] << 16);
    }
};

// Chunks whose bins begin elsewhere, the row's first being `off` bins above theirs: their
// counts are put where the row has their bins, and bins that it has not join the class
// on their side.  False if a chunk's own class on the other side would have to be told
// apart.
__device__ __forceinline__ bool into_line(ValueSmem& sm, const Anchor& an, Classes& cl, double part,
                                          int off, const ScratchCounts& count8) {
    constexpr int W = 8;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const uint64_t moved = __ballot(part > 0.0 && off != 0);
    if (moved == 0) return true;
    if (__ballot(part > 0.0 && off != 0 && (off > 0 ? cl.tail_n : cl.mid_n) != 0) != 0)
        return false;
    if (tid < 64) {
        sm.have[tid] = (uint32_t)off;
        sm.take[tid] = 0;
    }
    const int base = value_base((float)an.m), p0 = VB_PER * tid;
    // the least magnitude of the thread's bins, above the first one's
    const int mag0 = p0 < VB_SIDE ? VB_SIDE - VB_PER - p0 : p0 - VB_SIDE;
    __syncthreads();
#pragma unroll 1
    for (uint64_t rest = moved; rest != 0; rest &= rest - 1) {
        const int c = __builtin_ctzll(rest), o = (int)sm.have[c];
        uint64_t out[2] = {0, 0}, q[2] = {0, 0};
        if (o > 0 ? mag0 < o : mag0 >= VB_SIDE + o) count8(c, p0, out);
        if (mag0 + o >= 0 && mag0 + o < VB_SIDE) count8(c, p0 < VB_SIDE ? p0 - o : p0 + o, q);
        uint32_t n = 0;
        double sum = 0.0;
        if (__ballot((out[0] | out[1]) != 0) != 0) {
            uint32_t v = (uint32_t)(base - o + mag0) << 16 | (p0 < VB_SIDE ? 0u : 0x80000000u);
#pragma unroll 1
            for (int i = 0; i < VB_PER; ++i, v += 1u << 16) {
                const uint32_t ni = (uint32_t)out[0] & 0xFFFFu;
                const double w = an.weight(__uint_as_float(v));
                n += w > 0.0 ? ni : 0u;  // (what has no weight counts nowhere)
                sum += (double)ni * w;
                out[0] = out[0] >> 16 | out[1] << 48;
                out[1] >>= 16;
            }
            sum = group_sum<64>(sum);
            if (n != 0) atomicAdd(&sm.take[c], n);
        }
        if (lane == 0) sm.part[wv][c] = sum;
        // all have what they need of the chunk's counts
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        count8.replace(c, p0, q);
    }
    __syncthreads();
    if (moved >> lane & 1) {
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < W; ++v) sum += sm.part[v][lane];
        (off > 0 ? cl.mid : cl.tail) += sum;
        (off > 0 ? cl.mid_n : cl.tail_n) += sm.take[lane];
    }
    __syncthreads();
    return true;
}

// The row's end: the cuts, and the token.  It goes by count8 (see there) and the classes.
// hold(c): makes h hold chunk c, from index c * chunk on.  A cut that falls in a class
// needs LISTS: the row's elements of that class are listed and ranked among each other,
// unless there are too many.  False if it cannot be done.
template <bool LISTS, int R, typename Count8, typename Hold>
__device__ __forceinline__ bool values_cut(ValueSmem& sm, const Rule& r, const Anchor& an, int S,
                                           int64_t chunk, Classes cl, double part,
                                           Held<bf16_t, 8, R>& h, const Count8& count8,
                                           const Hold& hold, float* val, int32_t* idx) {
    constexpr int W = 8;
    auto& s = sm.s;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int base = value_base((float)an.m), p0 = VB_PER * tid;
    constexpr int AT_ONCE = 8;  // chunks whose counts are in flight, and held if these are all
    uint64_t held[AT_ONCE][2];
    const auto load_counts = [&](int c0) {
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            held[k][0] = held[k][1] = 0;
            if (c0 + k < S && lane_value(part, c0 + k < S ? c0 + k : 0) > 0.0)
                count8(c0 + k, p0, held[k]);
        }
    };
    const auto number = [&](int k, int j) {  // of position p0 + j in chunk k of those
        const int i = p0 < VB_SIDE ? VB_PER - 1 - j : j;
        return (uint32_t)((i < 4 ? held[k][0] : held[k][1]) >> (i % 4 * 16)) & 0xFFFFu;
    };
    // the bins of the row, their weights, and the classes
    Bins bin;
#pragma unroll
    for (int j = 0; j < VB_PER; ++j) bin.n[j] = 0;
#pragma unroll 1
    for (int c0 = 0; c0 < S; c0 += AT_ONCE) {
        load_counts(c0);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (c0 + k >= S) break;
#pragma unroll
            for (int j = 0; j < VB_PER; ++j) bin.n[j] += number(k, j);
        }
    }
    uint32_t count = 0;
    double mass = 0.0;
    bin.each([&](uint32_t n, double& w, int p) {
        w = n ? an.weight(position_value(p, base)) : 0.0;
        count += n;
        mass += (double)n * w;
    });
    const double mid = group_sum<64>(cl.mid), tail = group_sum<64>(cl.tail);
    const uint32_t mid_n = lane_value(wave_scan(cl.mid_n), 63);
    const uint32_t tail_n = lane_value(wave_scan(cl.tail_n), 63);
    // (units of 2^-48 lose the least weights of the classes, which a u at the very ends
    // of [0, 1] could still fall on)
    if ((mid_n != 0 || tail_n != 0) && (r.u < 0x1p-30 || r.u > 1.0 - 0x1p-30)) return false;
    // sums before each thread's bins; the middle class stands before position 2048
    const uint32_t cincl = wave_scan(count);
    const double mincl = wave_scan(mass);
    if (lane == 63) {
        s.wave32[wv] = cincl;
        s.waved[wv] = mincl;
    }
    if (tid == 0) s.found = VB_BINS;
    __syncthreads();
    uint32_t cbefore = cincl - count;
    double mbefore = lane_before(mincl), window = 0.0, positive = 0.0;
    uint32_t bins_n = 0, positive_n = 0;
#pragma unroll
    for (int v = 0; v < W; ++v) {
        if (v == wv) {
            cbefore += bins_n;
            mbefore += window;
        }
        if (v == W / 2) {
            positive = window;
            positive_n = bins_n;
        }
        bins_n += s.wave32[v];
        window += s.waved[v];
    }
    const bool behind = tid >= VB_SIDE / VB_PER;
    if (behind) {
        cbefore += mid_n;
        mbefore += mid;
    }
    __syncthreads();
    int cut = VB_BINS;          // position of the last kept value
    uint32_t keep = 0;          // elements of it that stay
    double all = window + mid + tail;
    enum { NONE, MIDDLE, TAIL };
    int split = NONE, listed = NONE;  // the class with a cut inside, and the listed one
    Cut inner = no_cut();
    const auto list_class = [&](int which) {
        if constexpr (!LISTS) return false;
        if (listed == which) return true;
        const uint32_t have = which == MIDDLE ? cl.mid_n : cl.tail_n;
        if ((which == MIDDLE ? mid_n : tail_n) > (uint32_t)VB_BINS) return false;
        listed = which;
        __syncthreads();
        if (tid == 0) s.n = 0;
        __syncthreads();
#pragma unroll 1
        for (uint64_t rest = __ballot(have != 0); rest != 0; rest &= rest - 1) {
            const int c = __builtin_ctzll(rest);
            hold(c);
            h.each([&](const u32x4& v, int32_t i) {
                uint32_t in = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t bits = pattern(v, e);
                    const bool middle = (bits & 0x7FFFu) < (uint32_t)base;
                    in |= value_bin(bits, (uint32_t)base) == (uint32_t)VB_BINS &&
                                  middle == (which == MIDDLE)
                              ? 1u << e
                              : 0u;
                }
                for (; __any(in != 0); in &= in - 1) {
                    const int e = in ? __builtin_ctz(in) : 0;
                    const uint32_t word = e < 2 ? v[0] : e < 4 ? v[1] : e < 6 ? v[2] : v[3];
                    const float x = __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16);
                    if (in && an.weight(x) > 0.0) {
                        const int j = atomicAdd(&s.n, 1);
                        if (j < VB_BINS) {
                            sm.lx[j] = x;
                            sm.li[j] = (uint32_t)(c * chunk) + (uint32_t)(i + e);
                        }
                    }
                }
            });
        }
        __syncthreads();
        return s.n > 0 && s.n <= VB_BINS;
    };
    const auto units = [&](float x) { return fixed48(an.weight(x)); };
    const auto inside = [&](int j) {
        return inner.keeps(sm.lx[j], sm.li[j]) && an.weight(sm.lx[j]) >= r.q;
    };
    const auto listed_sum = [&] {  // of what `inner` keeps, in units
        uint64_t v = 0;
        for (int j = tid; j < s.n; j += 64 * W)
            if (inner.keeps(sm.lx[j], sm.li[j])) v += units(sm.lx[j]);
        v = wave_total(v);
        if (lane == 0) s.wave64[wv] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) v += s.wave64[w];
        __syncthreads();
        return v;
    };
    const auto source = [&] {
        return ListSource{sm.lx, sm.li, s.n, (uint32_t)(S * chunk - 1)};
    };
    const uint32_t top = order_key((float)an.m), bottom = order_key(-__builtin_inff());
    if (r.k) {
        uint32_t b = cbefore;
        double d = mbefore;
        bin.each([&](uint32_t n, double w, int p) {
            if ((int64_t)b < r.k && r.k <= (int64_t)b + n) {
                s.found = p;
                s.above = (uint64_t)(r.k - b);
                s.base = d + (double)(r.k - b) * w;
            }
            b += n;
            d += (double)n * w;
        });
        __syncthreads();
        cut = s.found;
        if (cut < VB_BINS) {
            keep = (uint32_t)s.above;
            all = s.base;
        } else if (r.k <= (int64_t)bins_n + mid_n + tail_n) {
            // not among the bins: in the middle class, or beyond the end
            const int which = r.k <= (int64_t)bins_n + mid_n ? MIDDLE : TAIL;
            const int64_t k = r.k - (which == MIDDLE ? positive_n : bins_n + mid_n);
            if (!list_class(which)) return false;
            split = which;
            inner = find_cut<false>(s, source(), bottom, top, inner,
                                    (uint64_t)(k < s.n ? k : s.n), -1.0, units);
            all = (split == MIDDLE ? positive : window + mid) + (double)listed_sum() * 0x1p-48;
            if (split == MIDDLE) {
                cut = VB_SIDE - 1;
                keep = ~0u;
            }
        }
        __syncthreads();
    }
    if (r.p < 1.0) {
        const double target = r.p * all;
        if (tid == 0) s.found = VB_BINS;
        __syncthreads();
        double b = mbefore, b_at = 0.0, w_at = 0.0;
        uint32_t m_at = 0;
        int at = VB_BINS;
        // (the lowest position that reaches the target; the class in between is not one)
        bin.each([&](uint32_t n, double w, int p) {
            const uint32_t m = p < cut ? n : p == cut ? (n < keep ? n : keep) : 0u;
            const double a = b + (double)m * w;
            if (m != 0 && a >= target && at == VB_BINS) {
                at = p;
                b_at = b;
                w_at = w;
                m_at = m;
            }
            b = a;
        });
        if (at < VB_BINS) atomicMin(&s.found, at);
        __syncthreads();
        const bool mine = at == s.found;
        at = s.found;
        if (mine && at < VB_BINS) {
            const double need = __builtin_ceil((target - b_at) / w_at);
            uint32_t want = need >= 1.0 ? (need < (double)m_at ? (uint32_t)need : m_at) : 1;
            // (the quotient may be a step off: the smallest that reaches it)
            if (want > 1 && b_at + (double)(want - 1) * w_at >= target) --want;
            else if (want < m_at && b_at + (double)want * w_at < target) ++want;
            s.above = want;
        }
        __syncthreads();
        // or within a class: the one that stands before it, or beyond the end?
        const bool middle = split == MIDDLE ? at == VB_BINS
                                            : at >= VB_SIDE && cut >= VB_SIDE && mid_n != 0 &&
                                                  positive < target && positive + mid >= target;
        if (middle || (at == VB_BINS && tail_n != 0 && cut == VB_BINS)) {
            if (!list_class(middle ? MIDDLE : TAIL)) return false;
            split = middle ? MIDDLE : TAIL;
            const uint64_t sum = listed_sum();
            const double need =
                __builtin_ceil((target - (middle ? positive : window + mid)) * 0x1p48);
            const uint64_t want = need >= 1.0 ? (uint64_t)need : 1;
            if (sum == 0) return false;
            inner = find_cut<true>(s, source(), bottom, top, inner, want < sum ? want : sum, -1.0,
                                   units);
            if (middle) {
                cut = VB_SIDE - 1;
                keep = ~0u;
            }
        } else if (at < VB_BINS) {
            cut = at;
            keep = (uint32_t)s.above;
            split = NONE;
            inner = no_cut();
        }
        __syncthreads();
    }
    // min-p, and what stays of the classes
    bool mid_stays = split == MIDDLE || (mid_n != 0 && cut >= VB_SIDE);
    bool tail_stays = tail_n != 0 && cut == VB_BINS;
    if (r.q > 0.0) {
        const float tiny = __uint_as_float((uint32_t)base << 16);
        if (mid_stays) {
            const bool some = an.weight(tiny) >= r.q, every = an.weight(-tiny) >= r.q;
            if (some && !every && split != MIDDLE) {  // (so the tail stays out)
                if (!list_class(MIDDLE)) return false;
                split = MIDDLE;
                inner = no_cut();
            }
            mid_stays = some;
        }
        if (tail_stays) {
            tail_stays = an.weight(position_value(VB_BINS - 1, base)) >= r.q;
            if (tail_stays && split != TAIL) {
                if (!list_class(TAIL)) return false;
                split = TAIL;
            }
        }
        if (split == TAIL && !tail_stays) split = NONE;
        if (split == MIDDLE && !mid_stays) split = NONE;
    }
    if (split != NONE) {  // its kept weights by chunk, in the place of its whole ones
        __syncthreads();
        if (tid < 64) s.chunk[tid] = 0;
        __syncthreads();
        for (int j = tid; j < s.n; j += 64 * W)
            if (inside(j)) add_bin(s.chunk[sm.li[j] / (uint32_t)chunk], units(sm.lx[j]));
        __syncthreads();
        (split == MIDDLE ? cl.mid : cl.tail) = (double)s.chunk[lane] * 0x1p-48;
    }
    // the kept weights of each chunk
    bin.each([&](uint32_t, double& w, int p) {
        w = p > cut || w < r.q ? 0.0 : w;
        sm.weights[p < VB_SIDE ? VB_SIDE - 1 - p : p] = w;
    });
    const int at_cut = cut - p0;  // in [0, 8): this thread has the cut's bin
    uint32_t left = keep;
#pragma unroll 1
    for (int c0 = 0; c0 < S; c0 += AT_ONCE) {
        if (S > AT_ONCE) load_counts(c0);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (c0 + k >= S) break;
            double sum = 0.0;
            uint32_t have = 0;
#pragma unroll
            for (int j = 0; j < VB_PER; ++j) {
                const uint32_t n = number(k, j);
                sum += (double)n * bin.w[j];
                have = j == at_cut ? n : have;
            }
            if (at_cut >= 0 && at_cut < VB_PER) {
                const uint32_t take = have < left ? have : left;
                sm.have[c0 + k] = have;
                sm.take[c0 + k] = take;
                left -= take;
                double w = 0.0;
#pragma unroll
                for (int j = 0; j < VB_PER; ++j) w = j == at_cut ? bin.w[j] : w;
                sum -= (double)(have - take) * w;
            }
            sum = group_sum<64>(sum);
            if (lane == 0) sm.part[wv][c0 + k] = sum;
        }
    }
    __syncthreads();
    double kept = 0.0;  // of chunk `lane`
    if (lane < S) {
#pragma unroll
        for (int v = 0; v < W; ++v) kept += sm.part[v][lane];
        kept += (mid_stays ? cl.mid : 0.0) + (tail_stays ? cl.tail : 0.0);
    }
    const double incl = wave_scan(kept);
    const double total = lane_value(incl, 63), target = r.u * total;
    const uint64_t some = __ballot(kept > 0.0), past = __ballot(kept > 0.0 && incl > target);
    if (some == 0) return false;
    const int c = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
    const double rem = past ? target - (c ? lane_value(incl, c - 1) : 0.0) : __builtin_inf();
    hold(c);
    // of the elements that hold the cut's value, the chunk's first `take`
    const uint32_t i0 = (uint32_t)(c * chunk);
    uint32_t last = 0xFFFFFFFFu, partly = VB_BINS + 1;  // the bin that is cut within this chunk
    __syncthreads();
    if (cut < VB_BINS) {
        const uint32_t take = sm.take[c], have = sm.have[c];
        const int b = cut < VB_SIDE ? VB_SIDE - 1 - cut : cut;
        if (take == 0 && tid == 0) sm.weights[b] = 0.0;
        if (take != 0 && take != have) {
            const float v = position_value(cut, base);
            const bool ok = locate<true>(
                s, h,
                [&](const u32x4& q, uint32_t, double(&y)[8]) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = h.at(q, e) == v ? 1.0 : 0.0;
                },
                (double)take - 0.5, 1.0, 0, &sm.val, &sm.idx);
            __syncthreads();
            if (!ok) return false;
            last = (uint32_t)sm.idx;
            partly = (uint32_t)b;
        }
    }
    __syncthreads();
    const bool classes = mid_stays || tail_stays;
    return locate<true>(
        s, h,
        [&](const u32x4& q, uint32_t i, double(&y)[8]) {
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = value_bin(pattern(q, e), (uint32_t)base);
                const bool in = b < (uint32_t)VB_BINS && !(b == partly && i + e > last);
                const double x = sm.weights[b < (uint32_t)VB_BINS ? b : 0];
                y[e] = in ? x : 0.0;
                odd |= b == (uint32_t)VB_BINS;
            }
            if (classes && __any(odd)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t p = pattern(q, e);
                    const bool of = (p & 0x7FFFu) < (uint32_t)base ? mid_stays : tail_stays;
                    if (of && value_bin(p, (uint32_t)base) == (uint32_t)VB_BINS &&
                        inner.keeps(h.at(q, e), i0 + i + e)) {
                        const double w = an.weight(h.at(q, e));
                        y[e] = w >= r.q ? w : 0.0;
                    }
                }
            }
        },
        rem, total, i0, val, idx);
}

// The chunks of a row.
template <int R>
struct RowParts {
    const bf16_t* x;
    int64_t V, chunk;
    __device__ __forceinline__ void hold(int c, Held<bf16_t, 8, R>& h) const {
        const int64_t i0 = (int64_t)c * chunk;
        h.load(x + i0, (int32_t)(V - i0 < chunk ? V - i0 : chunk));
    }
};

// The same with lists, for the rows that need them (64 x 128256, a top-k among the 50
// elements next to 0 in every row: 82 us, by passes over memory 428; with a cut elsewhere
// 37).  In a function of its own: beside the common way its code and registers cost that 5%
// of 512 x 128256.
template <int R, typename Counts>
__device__ __attribute__((noinline)) bool values_lists(ValueSmem& sm, Rule r, float m, double c,
                                                       const bf16_t* x, int64_t V, int64_t chunk,
                                                       int S, Classes cl, double part,
                                                       Counts counts, float* val, int32_t* idx) {
    const Anchor an = anchor(m, c);
    const RowParts<R> row{x, V, chunk};
    Held<bf16_t, 8, R> h;
    __syncthreads();
    return values_cut<true>(sm, r, an, S, chunk, cl, part, h, counts,
                            [&](int c) { row.hold(c, h); }, val, idx);
}

}  // namespace osm
