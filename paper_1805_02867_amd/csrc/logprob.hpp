// Log probabilities of given tokens, the entropy and the best alternatives of rows (or chunks
// of rows) held in registers or streamed: one read of every element.
//
// What bounds them: large batches memory (2048 x 128256 bfloat16 with the entropy 86 us for 525
// MB, 6.1 TB/s, a plain read of as much 75.5; 300 x 32000 binary32 10.6 us for 38 MB, 8.3; 16385 x
// 1000 12.7 us for 66 MB, 12.3), short rows the arithmetic that is not their elements' (32768 x 32
// bfloat16 4.8 us), and a few rows the chain of a chunk and of the join (1 x 128256 5.1 us, with
// five alternatives 8.2).
//
// A row's state is (m, s, w) with c = log2(e) / temperature:
//   m = max x,
//   s = sum of 2^{(x_j - m) c} over all j but one that has x_j = m,
//   w = sum_j 2^{(x_j - m) c} (m - x_j) c,
// so that, in units of the natural logarithm, ln sum_j e^{x_j / T} = m / T + ln(1 + s) and the
// entropy is ln(1 + s) + ln(2) w / (1 + s).  s leaves one largest element out, since a trained
// model's token often has all the weight: in d = 1 + s a binary32 sum has lost what the others
// add, and ln p = -ln(1 + s) and 1 - p with it.  Terms of w are at least 0: nothing cancels.
// Two states merge as the online pair's do (Eq. 4), the smaller maximum's element joining the
// others:  with M = max, r = 2^{(m' - M) c} of the smaller one,
//   s = s + (s' + 1) r,   w = w + (w' + (M - m') c (s' + 1)) r.
// An empty state is (-inf, -1, 0): its s' + 1 is 0.
//
// Exponents.  A wavefront's are t = fma(x, c, -S) with S = m c rounded: one rounding of the
// difference, at any magnitude.  What S lacks, delta = m c - S (exact in an fma), is put right
// in its sums: with t = (x - m) c + delta, s is 2^-delta times the sum of 2^t, and so is w.  From
// |S| = 2^22 on delta would not be small: there the elements are replaced by x - m, and m by 0,
// ahead of the same loop.  (In the elements' type: where x - m rounds in bfloat16, x is so far
// from m that its weight is 0.)
#pragma once

#include "topk_held.hpp"
#include "wide.hpp"

namespace osm {

struct LogState {
    float m, s, w;
};

__device__ __forceinline__ LogState log_empty() { return {-__builtin_inff(), -1.0f, 0.0f}; }

__device__ __forceinline__ LogState log_merge(LogState a, LogState b, float c) {
    const bool first = a.m >= b.m || !(b.m == b.m);
    const LogState hi = first ? a : b, lo = first ? b : a;
    // (empty states are infinitely far: a bound keeps 0 times it 0)
    const float fall = __builtin_fminf((hi.m - lo.m) * c, 0x1p60f);
    const float r = exp2_hw(-fall), d = lo.s + 1.0f;
    return {hi.m, __builtin_fmaf(d, r, hi.s),
            __builtin_fmaf(__builtin_fmaf(fall, d, lo.w), r, hi.w)};
}

template <int STEP>
__device__ __forceinline__ LogState log_merge_step(LogState v, float c) {
    LogState a, b;
    bfly_operands<STEP>(v.m, a.m, b.m);
    bfly_operands<STEP>(v.s, a.s, b.s);
    bfly_operands<STEP>(v.w, a.w, b.w);
    return log_merge(a, b, c);
}

// Merge over the wavefront; lane 0's is the result (equal maxima make lanes differ by
// roundings).
__device__ __forceinline__ LogState log_merge_wave(LogState v, float c) {
    v = log_merge_step<0>(v, c);
    v = log_merge_step<1>(v, c);
    v = log_merge_step<2>(v, c);
    v = log_merge_step<3>(v, c);
    v = log_merge_step<4>(v, c);
    v = log_merge_step<5>(v, c);
    return {lane_value(v.m, 0), lane_value(v.s, 0), lane_value(v.w, 0)};
}

// Below this exponent a weight is 0 (v_exp_f32 gives no subnormals): it stands for all of them
// in w, where -inf times 0 would be no number.
constexpr float kLogFloor = -200.0f;

// Adds the weights of a vector, and (ENT) minus their falls.  SKIP: an element of value m is
// left out, the first.
template <bool ENT, bool SKIP, int E>
__device__ __forceinline__ void log_add(const float (&x)[E], float m, float c, float S, float& s,
                                        float& w) {
    bool done = !SKIP;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float t = __builtin_fmaf(x[e], c, -S);
        float p = exp2_hw(t);
        if constexpr (SKIP) {
            const bool is = !done && x[e] == m;
            p = is ? 0.0f : p;
            done = done || is;
        }
        s += p;
        if constexpr (ENT) w = __builtin_fmaf(p, __builtin_fmaxf(t, kLogFloor), w);
    }
}

// The largest of a vector of bfloat16 elements as integers of 16 bits: the largest element if
// that is not negative, else some negative number.
__device__ __forceinline__ int signed_max(u32x4 q) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const s16x2 a = __builtin_elementwise_max(__builtin_bit_cast(s16x2, (uint32_t)q.x),
                                              __builtin_bit_cast(s16x2, (uint32_t)q.y));
    const s16x2 b = __builtin_elementwise_max(__builtin_bit_cast(s16x2, (uint32_t)q.z),
                                              __builtin_bit_cast(s16x2, (uint32_t)q.w));
    const s16x2 c = __builtin_elementwise_max(a, b);
    return c.x > c.y ? c.x : c.y;
}

// x - m in the elements' type.
template <typename T>
__device__ __forceinline__ u32x4 less(u32x4 q, float m) {
    float v[Vec<T>::N];
    widen<T>(q, v);
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) v[e] -= m;
    if constexpr (Vec<T>::N == 8)
        return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                     pack_bf16x2(v[6], v[7])};
    else
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                     __float_as_uint(v[3])};
}

// What lane l < T of a wavefront knows of its row's l-th token.  The index is asked for ahead of
// the row, the element behind it: neither is waited for then.
struct LogToken {
    int32_t i = -1;
    float x = 0.0f;
    bool in = false;

    __device__ __forceinline__ void index(const LogprobRows& a, int64_t row, int lane) {
        if (a.T > 0) i = a.tokens[row * a.T + (lane < a.T ? lane : 0)];
    }
    template <typename T>
    __device__ __forceinline__ void element(const LogprobRows& a, const T* xr, int lane) {
        if (a.T > 0) {
            in = lane < a.T && i >= 0 && (int64_t)i < a.V;
            x = load1(xr + (in ? i : 0));
        }
    }
};

// What a row's alternatives need of its state.
struct LogEnd {
    double m, ln_d;
    bool good;
};

__device__ __forceinline__ LogEnd log_end_of(const LogState& v) {
    return {(double)v.m, ln_1p(v.s), __builtin_fabsf(v.m) < __builtin_inff() && v.s == v.s};
}

// log p of an element.
__device__ __forceinline__ float log_of(const LogprobRows& a, const LogEnd& v, float x) {
    const float lp = (float)(((double)x - v.m) * a.inverse - v.ln_d);
    return v.good ? lp : __builtin_nanf("");
}

// A row's entropy and state, by lane 0.
__device__ __forceinline__ void log_store_row(const LogprobRows& a, int64_t row, const LogState& v,
                                              const LogEnd& end, int lane) {
    if (lane != 0) return;
    const float nan = __builtin_nanf("");
    if (a.entropy) {
        const double d = 1.0 + (double)v.s, q = (double)__builtin_amdgcn_rcpf((float)d);
        const double h = end.ln_d + 0.69314718055994530942 * (double)v.w * (q * (2.0 - d * q));
        a.entropy[row] = end.good ? (float)h : nan;
    }
    if (a.stats) {
        a.stats[row * 2] = end.good ? v.m : nan;
        a.stats[row * 2 + 1] = end.good ? v.s : nan;
    }
}

// A row's outputs but for the alternatives, by one wavefront, from its state and lane l's token.
__device__ __forceinline__ LogEnd log_store(const LogprobRows& a, int64_t row, const LogState& v,
                                            const LogToken& t) {
    const int lane = threadIdx.x & 63;
    const LogEnd end = log_end_of(v);
    if (lane < a.T) a.logp[row * a.T + lane] = t.in ? log_of(a, end, t.x) : 0.0f;
    log_store_row(a, row, v, end, lane);
    return end;
}

// Lane l has the l-th alternative.
__device__ __forceinline__ void log_store_top(const LogprobRows& a, int64_t row, LogEnd v,
                                              uint64_t key) {
    const int lane = threadIdx.x & 63;
    if (lane >= a.K) return;
    a.top_vals[row * a.K + lane] = log_of(a, v, key_value(key));
    a.top_idx[row * a.K + lane] = v.good ? key_index(key) : -1;
}

// LDS of a workgroup.
template <int W, bool SEL>
struct LogSmem {
    LogState state[W];
    LogEnd end;
    bool last;
    HeldSmem<W> top;
};
template <int W>
struct LogSmem<W, false> {
    LogState state[W];
};

// A chunk's partial in scratch: its state, as two 64-bit words that are stored and read at
// the device's coherence point.
__device__ __forceinline__ void log_put(uint64_t* p, LogState v) {
    const uint64_t ms = (uint64_t)__float_as_uint(v.s) << 32 | __float_as_uint(v.m);
    __hip_atomic_store(p, ms, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(p + 1, (uint64_t)__float_as_uint(v.w), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ LogState log_get(const uint64_t* p) {
    const uint64_t ms = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint64_t w = __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return {__uint_as_float((uint32_t)ms), __uint_as_float((uint32_t)(ms >> 32)),
            __uint_as_float((uint32_t)w)};
}

// Leaves chunk vr's state at the device's coherence point, by one wavefront, then counts it:
// whether it is the row's last.
__device__ __forceinline__ bool log_arrive(const LogprobSplit& p, int64_t vr, uint32_t in_launch,
                                           LogState v) {
    const int lane = threadIdx.x & 63;
    if (lane == 0) log_put(p.states + vr * 2, v);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    uint32_t done = 0;
    if (lane == 0)
        done = __hip_atomic_fetch_add(p.ctr + in_launch, 1u, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
    return __builtin_amdgcn_readfirstlane(done) == (uint32_t)p.S - 1;
}

// The state of a row whose chunks are all in, by one wavefront; its count is left at 0.
__device__ __forceinline__ LogState log_join(const LogprobSplit& p, uint32_t in_launch, float c) {
    const int lane = threadIdx.x & 63;
    const int64_t first = (int64_t)in_launch * p.S;
    LogState v = log_empty();
    for (int j = lane; j < p.S; j += 64) v = log_merge(v, log_get(p.states + (first + j) * 2), c);
    v = log_merge_wave(v, c);
    if (lane == 0)
        __hip_atomic_store(p.ctr + in_launch, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return v;
}

// The end of a workgroup's row or (PART) chunk: its wavefronts' states and (SEL) lists are in
// LDS.  The chunk that completes a row merges it.
template <typename T, int W, bool SEL, bool PART>
__device__ __forceinline__ void log_end(const LogprobRows& a, const LogprobSplit& p,
                                        LogSmem<W, SEL>& sm, int64_t row, uint32_t in_launch,
                                        int64_t vr, LogToken tok) {
    constexpr uint32_t GRAN = Vec<T>::N == 8 ? 1u << 16 : 1u;
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float c = a.c;
    auto state = [&] {
        LogState v = sm.state[0];
#pragma unroll
        for (int i = 1; i < W; ++i) v = log_merge(v, sm.state[i], c);
        return v;
    };
    if constexpr (!SEL) {
        if (wv != 0) return;
        LogState v = state();
        if constexpr (PART) {
            if (!log_arrive(p, vr, in_launch, v)) return;
            v = log_join(p, in_launch, c);
        }
        log_store(a, row, v, tok);
    } else {
        uint64_t key = 0;
        if (wv == 0) key = held_finish<W>(sm.top.list, sm.top.cnt, a.K);
        if constexpr (PART) {
            // the partial, at the device's coherence point; then the row's count
            if (wv == 0) {
                if (lane < a.K)
                    __hip_atomic_store(p.keys + vr * a.K + lane, key, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
                const bool last = log_arrive(p, vr, in_launch, state());
                if (lane == 0) sm.last = last;
            }
            __syncthreads();
            if (!sm.last) return;
            // every chunk of the row is in; a merge of more partial keys than one wavefront
            // holds takes them all
            const int64_t n = (int64_t)p.S * a.K;
            const uint64_t* pk = p.keys + (int64_t)in_launch * n;
            MD none;
            if (n > 64 * TK_MERGE_B)
                held_merge<TK_VALUES, W, TK_MERGE_B, GRAN, true>(sm.top, wv, pk, nullptr, n, 0,
                                                                 a.K, &key, &none);
            else if (wv == 0)
                held_merge<TK_VALUES, 1, TK_MERGE_B, GRAN, true>(sm.top, 0, pk, nullptr, n, 0,
                                                                 a.K, &key, &none);
        }
        if (wv == 1) {
            LogState v;
            if constexpr (PART) v = log_join(p, in_launch, c);
            else v = state();
            const LogEnd end = log_store(a, row, v, tok);
            if (lane == 0) sm.end = end;
        }
        __syncthreads();
        if (wv == 0) log_store_top(a, row, sm.end, key);
    }
}

// Wavefronts per SIMD asked of the compiler.
template <typename T, int W, int R, bool SEL, bool PART>
constexpr int log_waves() {
    constexpr bool bf = Vec<T>::N == 8;
    if (SEL && R >= 6) return R > 12 ? 4 : R > 8 ? (bf ? 4 : 5) : R > 6 ? (bf ? 6 : 7) : 7;
    return held_waves<T, W, R, PART>();
}

// Rows (PART = false: from row0 on) or chunks of rows (PART = true: workgroup b has chunk b % S of
// row row0 + b / S) of at most 64 W R whole 16-byte vectors, W wavefronts each (W = 1: four rows a
// workgroup).  SEL: with alternatives, selected as topk_held.hpp does.  ENT: with w.
template <typename T, int W, int R, bool SEL, bool ENT, bool PART>
__global__
__launch_bounds__(W == 1 ? TK_BLOCK : 64 * W, (log_waves<T, W, R, SEL, PART>())) void logprob_held(
    const LogprobRows a, const LogprobSplit p) {
    static_assert(!PART || W > 1, "chunks take a workgroup each");
    constexpr int E = Vec<T>::N, TR = 64 * W;
    constexpr uint32_t GRAN = E == 8 ? 1u << 16 : 1u;
    __shared__ LogSmem<W, SEL> sm;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tr = W == 1 ? lane : tid;
    const int64_t vr = W == 1 ? (int64_t)blockIdx.x * (TK_BLOCK / 64) + wv : (int64_t)blockIdx.x;
    if (W == 1 && vr >= p.rows) return;  // whole wavefronts; no barrier follows
    const uint32_t in_launch = PART ? blockIdx.x / (uint32_t)p.S : 0;
    const int64_t row = p.row0 + (PART ? in_launch : vr);
    const int64_t start = PART ? (blockIdx.x - in_launch * (uint32_t)p.S) * p.chunk : 0;
    const int64_t left = a.V - start;
    const T* xr = static_cast<const T*>(a.x) + row * a.ld;
    const HeldSpan<T> sp(xr, 0, start, 0, (int)(PART && p.chunk < left ? p.chunk : left));
    const int nvec = sp.nvec;
    const float ninf = -__builtin_inff(), c = a.c;

    LogToken tok;
    // with alternatives the second wavefront has the row's state while the first one sorts them
    constexpr int OWN = SEL ? 1 : 0;
    if (wv == OWN || W == 1) tok.index(a, row, lane);
    // all loads first; lanes past the row load its last vector and mask it
    u32x4 buf[R];
    auto load = [&] {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int v = tr + i * TR;
            buf[i] = __builtin_nontemporal_load(sp.vb + (v < nvec ? v : nvec - 1));
        }
    };
    if (nvec > 0) {
        load();
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) buf[i] = u32x4{0, 0, 0, 0};
    }
    const float ex = tr < sp.ne ? load1(sp.xr + sp.extra(tr)) : ninf;
    if (wv == OWN || W == 1) tok.element(a, xr, lane);

    // 1. maxima by vector, and the wavefront's.  bfloat16 ones by two elements at a time as
    // integers, which order numbers that are not negative: where the wavefront has one, and only
    // the largest is asked for, that is all.
    float vm[R], lm = __builtin_fmaxf(ex, ninf), wm;  // a NaN element gives -inf
    constexpr bool FAST = E == 8 && !SEL;
    if constexpr (FAST) {
        int im = (int)__float_as_uint(ex) >> 16;  // (negative for -0.0 as well)
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int v = tr + i * TR < nvec ? signed_max(buf[i]) : -1;
            vm[i] = __uint_as_float((uint32_t)v << 16);
            im = v > im ? v : im;
        }
        wm = __builtin_amdgcn_ballot_w64(im >= 0) != 0
                 ? wave_max_f(im >= 0 ? __uint_as_float((uint32_t)im << 16) : ninf)
                 : ninf;
    }
    if (!FAST || !(wm > ninf)) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            opaque(buf[i]);
            vm[i] = tr + i * TR < nvec ? held_vmax<T, TK_VALUES>(buf[i]) : ninf;
            lm = max3_raw(lm, vm[i], ninf);
        }
        wm = wave_max_f(lm);
    }
    // 2. the wavefront's state.  The element that is left out: the head or tail element of
    // the first lane that has the maximum there, else in that lane's vector `left_out`, which is
    // looked at again by itself.
    LogState st;
    {
        float m = wm > ninf ? wm : 0.0f;  // (no elements, or only -inf)
        float s = 0.0f, w = 0.0f, x1[1] = {ex};
        const uint64_t at_ex = __builtin_amdgcn_ballot_w64(ex == m);
        uint64_t owner = at_ex;
        int left_out = -1;
        if (at_ex == 0) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const uint64_t has = __builtin_amdgcn_ballot_w64(vm[i] == m);
                const bool here = left_out < 0 && has != 0;
                owner = here ? has : owner;
                left_out = here ? i : left_out;
            }
        }
        const bool mine = wm > ninf && owner != 0 && lane == __builtin_ctzll(owner | 1ull << 63);
        const bool far = __builtin_fabsf(m * c) >= 0x1p22f;
        if (rare(far)) {
            x1[0] -= m;
#pragma unroll
            for (int i = 0; i < R; ++i) buf[i] = less<T>(buf[i], m);
            m = 0.0f;
        }
        const float S = m * c, delta = __builtin_fmaf(m, c, -S);
        if (!(mine && at_ex != 0)) log_add<ENT, false>(x1, m, c, S, s, w);
        u32x4 again = buf[0];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            opaque(buf[i]);
            if (i == 0 || i * TR < nvec) {  // uniform
                float xv[E], ps = 0.0f, pw = 0.0f;
                widen<T>(buf[i], xv);
                log_add<ENT, false>(xv, m, c, S, ps, pw);
                bool counts = tr + i * TR < nvec;
                if (i == left_out) {  // uniform
                    again = buf[i];
                    counts = counts && !mine;
                }
                s += counts ? ps : 0.0f;
                if constexpr (ENT) w += counts ? pw : 0.0f;
            }
        }
        if (left_out >= 0) {
            float xv[E], ps = 0.0f, pw = 0.0f;
            widen<T>(again, xv);
            log_add<ENT, true>(xv, m, c, S, ps, pw);
            s += mine ? ps : 0.0f;
            if constexpr (ENT) w += mine ? pw : 0.0f;
        }
        s = group_sum<64>(s);
        const float back = exp2_hw(-delta);
        if constexpr (ENT) w = back * __builtin_fmaf(delta, s, -group_sum<64>(w));
        s *= back;
        st = LogState{wm, wm > ninf ? s : s - 1.0f, w};
        if (SEL && rare(far) && nvec > 0) load();
    }
    uint64_t key = 0;
    if constexpr (SEL) {
        // 3. the candidates: elements at or above a threshold from the lanes' maxima (steps 2
        // and 3 of topk_held.hpp)
        const int K = a.K;
        KthBound b;
        if constexpr (W == 1) {
            constexpr int G = R == 1 ? 2 : R < 4 ? R : 4;
            float gm[G];
#pragma unroll
            for (int g = 0; g < G; ++g) gm[g] = g == 0 ? __builtin_fmaxf(ex, ninf) : ninf;
            if constexpr (R == 1) {
                float xv[E];
                widen<T>(buf[0], xv);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    gm[e % 2] = __builtin_fmaxf(gm[e % 2], tr < nvec ? xv[e] : ninf);
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i) gm[i % G] = max3_raw(gm[i % G], vm[i], ninf);
            }
            uint32_t g[G];
#pragma unroll
            for (int i = 0; i < G; ++i) g[i] = order_word(gm[i]);
            b = kth_bound<G, GRAN>(g, order_word(wm), K);
        } else {
            b = team_bound<W, GRAN>(sm.top, order_word(lm), K);
        }
        HeldList hl{sm.top.list[wv], K, 0, 0ull};
        float th = key_value((uint64_t)b.lo << 32);
        uint32_t hm = (uint32_t)(tr < sp.ne && ex >= th) << R;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            opaque(buf[i]);
            hm |= (uint32_t)(tr + i * TR < nvec && vm[i] >= th) << i;
        }
        if (rare(b.tied && nvec >= K)) {
            const float up = key_value((uint64_t)b.up << 32);
            if (held_ties<T, W, R>(sm.top, hl, sp, buf, tr, th, up)) {
                th = up;
                hm &= 1u << R;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    opaque(buf[i]);
                    const float v = held_vmax<T, TK_VALUES>(buf[i]);
                    hm |= (uint32_t)(tr + i * TR < nvec && v >= th) << i;
                }
            }
        }
        held_offer<T, R, TR>(hl, sp, buf, tr, hm, th, ex);
        if constexpr (W == 1) {
            wave_sync();
            key = held_finish<1>(&sm.top.list[wv], &hl.n, K);
        } else if (lane == 0) {
            sm.top.cnt[wv] = hl.n;
        }
    }
    // 4. the row's outputs, or the chunk's partial
    if constexpr (W == 1) {
        const LogEnd end = log_store(a, row, st, tok);
        if constexpr (SEL) log_store_top(a, row, end, key);
    } else {
        if (lane == 0) sm.state[wv] = st;
        __syncthreads();
        log_end<T, W, SEL, PART>(a, p, sm, row, in_launch, vr, tok);
    }
}

// ------------------------------------------------------------------ short rows
// Rows of at most TL R whole vectors by TL lanes each, 64 / TL rows a wavefront: what a row costs
// besides its elements is shared between them.  The element that s leaves out is the first one of
// the first lane that has the maximum, found as it is added.
template <typename T, bool ENT, int TL, int R>
__global__ __launch_bounds__(TK_BLOCK) void logprob_short(const LogprobRows a,
                                                          const LogprobSplit p) {
    constexpr int E = Vec<T>::N, ROWS = TK_BLOCK / TL;
    const int lane = threadIdx.x % TL, at = threadIdx.x & 63;
    const uint64_t team = ((1ull << TL) - 1) << (at / TL * TL);
    const float ninf = -__builtin_inff(), c = a.c;
    // rows behind the last one do that again, and store nothing
    const int64_t vr = (int64_t)blockIdx.x * ROWS + threadIdx.x / TL;
    const bool live = vr < p.rows;
    const int64_t row = p.row0 + (live ? vr : p.rows - 1);
    const T* xr = static_cast<const T*>(a.x) + row * a.ld;
    const HeldSpan<T> sp(xr, 0, 0, 0, (int)a.V);
    const int nvec = sp.nvec;
    int32_t tok = a.T > 0 ? a.tokens[row * a.T + (lane < a.T ? lane : 0)] : -1;
    u32x4 buf[R];
    const uint32_t low = E == 8 ? 0xFF80FF80u : 0xFF800000u;
#pragma unroll
    for (int i = 0; i < R; ++i) buf[i] = u32x4{low, low, low, low};
    if (nvec > 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int v = lane + i * TL;
            buf[i] = __builtin_nontemporal_load(sp.vb + (v < nvec ? v : nvec - 1));
        }
    }
    float ex = lane < sp.ne ? load1(xr + sp.extra(lane)) : ninf;
    auto inside = [&](int32_t t) { return t >= 0 && (int64_t)t < a.V; };
    float tx = a.T > 0 ? load1(xr + (inside(tok) ? tok : 0)) : 0.0f;
    float lm = __builtin_fmaxf(ex, ninf);  // a NaN element gives -inf
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool in = lane + i * TL < nvec;
        buf[i] = u32x4{in ? buf[i].x : low, in ? buf[i].y : low, in ? buf[i].z : low,
                       in ? buf[i].w : low};
        opaque(buf[i]);
        lm = max3_raw(lm, held_vmax<T, TK_VALUES>(buf[i]), ninf);
    }
    const float wm = group_max<TL>(lm);
    const uint64_t who = __builtin_amdgcn_ballot_w64(lm == wm) & team;
    bool done = at != __builtin_ctzll(who | 1ull << 63) || !(wm > ninf);
    float m = wm > ninf ? wm : 0.0f;  // (no elements, or only -inf)
    if (rare(__builtin_amdgcn_ballot_w64(__builtin_fabsf(m * c) >= 0x1p22f) != 0)) {
        const bool far = __builtin_fabsf(m * c) >= 0x1p22f;
        const float by = far ? m : 0.0f;
        ex -= by;
#pragma unroll
        for (int i = 0; i < R; ++i) buf[i] = less<T>(buf[i], by);
        m -= by;
    }
    const float S = m * c, delta = __builtin_fmaf(m, c, -S);
    float s = 0.0f, w = 0.0f;
    auto add = [&](float x) {
        const float t = __builtin_fmaf(x, c, -S);
        const bool is = !done && x == m;
        done = done || is;
        const float q = is ? 0.0f : exp2_hw(t);
        s += q;
        if constexpr (ENT) w = __builtin_fmaf(q, __builtin_fmaxf(t, kLogFloor), w);
    };
    add(ex);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        opaque(buf[i]);
        float xv[E];
        widen<T>(buf[i], xv);
#pragma unroll
        for (int e = 0; e < E; ++e) add(xv[e]);
    }
    s = group_sum<TL>(s);
    const float back = exp2_hw(-delta);
    if constexpr (ENT) w = back * __builtin_fmaf(delta, s, -group_sum<TL>(w));
    s *= back;
    LogState st{wm, wm > ninf ? s : s - 1.0f, w};
    const LogEnd end = log_end_of(st);
    if (!live) return;
    log_store_row(a, row, st, end, lane);
    for (int i = lane; i < a.T; i += TL) {
        if (i != lane) {
            tok = a.tokens[row * a.T + i];
            tx = load1(xr + (inside(tok) ? tok : 0));
        }
        a.logp[row * a.T + i] = inside(tok) ? log_of(a, end, tx) : 0.0f;
    }
}

// ------------------------------------------------------------------ streamed rows
// Rows or chunks by a workgroup of W wavefronts that stream them, U vectors a lane on their
// way while as many are worked on: memory is never left waiting for a reduction, which rows held
// in registers do between their loads.
//
// A wavefront's reference is its own maximum so far: one comparison a step finds whether that
// changes (of bfloat16 elements as integers of 16 bits, where the maximum is not negative).  Each
// lane sums all of its elements.  The one that s leaves out has weight 1 in its lane's sum; where
// the others of the wavefront add less than that, that lane's elements are read once more at the
// end, the largest apart, by the whole wavefront.
constexpr int LS_U = 4;  // vectors of a step

template <typename T, bool ENT>
struct LogStream {
    static constexpr int E = Vec<T>::N;
    float c;
    float m = -__builtin_inff();   // the wavefront's maximum
    float lm = -__builtin_inff();  // this lane's, where it is the wavefront's
    float S = 0.0f;                // m c, rounded
    float d = 0.0f, w = 0.0f;      // this lane's sums, relative to S
    bool far = false;              // |m c| has reached 2^22

    static __device__ __forceinline__ u32x4 nothing() {
        const uint32_t v = E == 8 ? 0xFF80FF80u : 0xFF800000u;
        return u32x4{v, v, v, v};
    }
    // The largest element of a step, if that is above the maximum or from `th` on (inf: no such
    // line).  As integers -0.0 is below all other elements: it is not above a maximum from 0 on,
    // but it reaches a line at 0.
    template <int U>
    __device__ __forceinline__ float largest(const u32x4 (&q)[U], float th) const {
        if constexpr (E == 8) {
            if (m >= 0.0f && th > 0.0f) {
                int v = -1;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = signed_max(q[u]);
                    v = i > v ? i : v;
                }
                return __uint_as_float((uint32_t)v << 16);  // (NaN for -1)
            }
        }
        float v = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            u32x4 t = q[u];
            if (E == 8) opaque(t);  // (or it is widened ahead of the test above)
            v = max3_raw(v, held_vmax<T, TK_VALUES>(t), v);
        }
        return v;
    }
    // (returns that largest element)
    template <int U>
    __device__ __forceinline__ float step(const u32x4 (&q)[U], float th) {
        const float v = largest(q, th);
        lm = v > lm ? v : lm;
        if (rare(__builtin_amdgcn_ballot_w64(v > m) != 0)) {
#pragma clang fp contract(off)  // (the step between the references as they are, both rounded)
            const float top = wave_max_f(lm), S2 = top * c, fall = S - S2;
            if (m > -__builtin_inff()) {
                const float r = exp2_hw(fall);
                if constexpr (ENT) w = r * __builtin_fmaf(fall, d, w);
                d *= r;
            } else if constexpr (ENT) {
                w = d;  // 0, or NaN
            }
            m = top;
            S = S2;
            far = far || !(__builtin_fabsf(S2) < 0x1p22f);
        }
        float ps = 0.0f, pw = 0.0f;  // (a step's apart: the chain of roundings is a tenth as long)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[E];
            widen<T>(q[u], x);
            log_add<ENT, false>(x, 0.0f, c, S, ps, pw);
        }
        d += ps;
        if constexpr (ENT) w += pw;
        return v;
    }
    // The wavefront's state.  ex: the lane's head or tail element; the others are its vectors
    // first + lane, first + lane + stride, ... of n from vb.
    __device__ __forceinline__ LogState end(float ex, const u32x4* vb, int first, int stride,
                                            int n) const {
        const int lane = threadIdx.x & 63;
        if (!(m > -__builtin_inff())) return {m, group_sum<64>(d) - 1.0f, 0.0f};
        const float delta = __builtin_fmaf(m, c, -S), one = exp2_hw(delta);
        const uint64_t who = __builtin_amdgcn_ballot_w64(lm == m);
        const int owner = who != 0 ? __builtin_ctzll(who) : 0;
        const bool mine = lane == owner;
        const float rest = group_sum<64>(mine ? 0.0f : d);
        // (the one's own exponent is delta)
        float s = rest + (lane_value(d, owner) - one);
        float fall = __builtin_fmaf(-delta, one, group_sum<64>(w));
        if (s < 1.0f) {
            float ps = 0.0f, pw = 0.0f;
            const float oex = lane_value(ex, owner);
            bool out = oex == m;
            if (!out && lane == 0) {
                const float x1[1] = {oex};
                log_add<ENT, false>(x1, m, c, S, ps, pw);
            }
            for (int i = first + owner; i < n; i += 64 * stride) {
                const int v = i + lane * stride;
                float x[E], top = -__builtin_inff();
                widen<T>(v < n ? vb[v] : nothing(), x);
#pragma unroll
                for (int e = 0; e < E; ++e) top = __builtin_fmaxf(top, x[e]);
                const uint64_t has = __builtin_amdgcn_ballot_w64(top == m);
                if (!out && has != 0 && lane == __builtin_ctzll(has | 1ull << 63))
                    log_add<ENT, true>(x, m, c, S, ps, pw);
                else
                    log_add<ENT, false>(x, m, c, S, ps, pw);
                out = out || has != 0;
            }
            s = rest + group_sum<64>(ps);
            fall = group_sum<64>(mine ? 0.0f : w) + group_sum<64>(pw);
        }
        const float r = exp2_hw(-delta);
        return {m, s * r, ENT ? r * __builtin_fmaf(delta, s, -fall) : 0.0f};
    }
};

// A vector's state by one lane, whatever its magnitude.
template <typename T>
__device__ __forceinline__ LogState log_of_vector(u32x4 q, float c) {
    constexpr int E = Vec<T>::N;
    float x[E];
    widen<T>(q, x);
    const float m = held_vmax<T, TK_VALUES>(q), at = m > -__builtin_inff() ? m : 0.0f;
    LogState v{m, 0.0f, 0.0f};
    bool done = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float t = (x[e] - at) * c;
        const bool is = !done && x[e] == m;
        done = done || is;
        const float p = is && m > -__builtin_inff() ? 0.0f : exp2_hw(t);
        v.s += p;
        v.w = __builtin_fmaf(p, -__builtin_fmaxf(t, kLogFloor), v.w);
    }
    if (!(m > -__builtin_inff())) v.s -= 1.0f;
    return v;
}

// The alternatives of a streamed row or chunk.  `th` is a value that K elements of the team's
// first step reach.  Where a step has elements of at least that, only the lanes that have them are
// noted; at the end, when the K-th largest of the lanes' maxima bounds the result far better, the
// vectors of the few whose largest element reaches it are read once more, and their elements
// offered to the wavefront's list (HeldList, topk_held.hpp).
template <typename T, int W>
struct LogPicks {
    static constexpr int E = Vec<T>::N, TR = 64 * W, U = LS_U;
    static constexpr uint32_t GRAN = E == 8 ? 1u << 16 : 1u;
    HeldList hl;
    uint64_t* notes;  // TH_LIST of them: image of the lane's largest element, step * 64 + lane
    int n;            // noted (wave-uniform), at most TH_CUT between steps
    float th;         // smaller elements are not among the K largest
    float th0;        // nor are such head and tail elements
    float lm;         // the lane's largest element, where that is at least th

    static __device__ __forceinline__ float word_value(uint32_t w) {
        return key_value((uint64_t)w << 32);
    }
    // From the first step's vectors (those behind the last one are not looked at) and the lanes'
    // head or tail elements, by the whole workgroup.
    __device__ __forceinline__ void begin(HeldSmem<W>& sm, uint64_t* mine, int wv, int K,
                                          const HeldSpan<T>& sp, const u32x4 (&q)[U], float ex) {
        const int tr = threadIdx.x;
        hl = HeldList{sm.list[wv], K, 0, 0ull};
        notes = mine;
        n = 0;
        lm = __builtin_fmaxf(ex, -__builtin_inff());
#pragma unroll
        for (int u = 0; u < U; ++u) {
            u32x4 t = q[u];
            opaque(t);
            if (tr + u * TR < sp.nvec) lm = __builtin_fmaxf(lm, held_vmax<T, TK_VALUES>(t));
        }
        const KthBound b = team_bound<W, GRAN>(sm, order_word(lm), K);
        th = th0 = word_value(b.lo);
        if (rare(b.tied && sp.nvec >= K)) {
            // (equal head elements, ahead of the ties in vectors, are offered at the end)
            const float up = word_value(b.up);
            if (held_ties<T, W, U>(sm, hl, sp, q, tr, th, up)) th = up;
        }
    }
    // v: the lane's largest element of step k, where that is at least th.
    __device__ __forceinline__ void step(const HeldSpan<T>& sp, int k, float v) {
        const uint64_t who = __builtin_amdgcn_ballot_w64(v >= th);
        if (who == 0) return;
        const int lane = threadIdx.x & 63;
        const uint32_t below = __builtin_amdgcn_mbcnt_hi(
            (uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
        if (v >= th) notes[n + below] = (uint64_t)order_word(v) << 32 | (uint32_t)(k * 64 + lane);
        n += __builtin_popcountll(who);
        lm = __builtin_fmaxf(lm, v);
        if (rare(n > TH_CUT)) {
            const uint32_t g[1] = {order_word(lm)};
            th = __builtin_fmaxf(th, word_value(kth_bound<1, GRAN>(g, wave_hi(g), hl.K).lo));
            keep();
            if (n > TH_CUT) look(sp);
        }
    }
    // Only the notes that reach th stay.
    __device__ __forceinline__ void keep() {
        const int lane = threadIdx.x & 63, had = n;
        const uint32_t t = order_word(th);
        uint64_t k[3];
        wave_sync();
#pragma unroll
        for (int j = 0; j < 3; ++j) k[j] = lane + 64 * j < had ? notes[lane + 64 * j] : 0ull;
        wave_sync();
        n = 0;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const bool p = lane + 64 * j < had && (uint32_t)(k[j] >> 32) >= t;
            const uint64_t mask = __builtin_amdgcn_ballot_w64(p);
            const uint32_t below = __builtin_amdgcn_mbcnt_hi(
                (uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
            if (p) notes[n + below] = k[j];
            n += __builtin_popcountll(mask);
        }
        wave_sync();
    }
    // The elements of at least th of the noted lanes' vectors go to the list.
    __device__ __forceinline__ void look(const HeldSpan<T>& sp) {
        const int lane = threadIdx.x & 63, first = (threadIdx.x & ~63);
        wave_sync();
        for (int i = 0; i < n; i += 64 / U) {
            const int at = i + lane / U;
            const uint32_t note = at < n ? (uint32_t)notes[at] : 0;
            const int64_t v64 = (int64_t)(note >> 6) * (TR * U) + (lane % U) * TR + first +
                                (int)(note & 63);
            const bool in = at < n && v64 < sp.nvec;
            const int v = in ? (int)v64 : 0;
            u32x4 q[1] = {sp.vb[v]};
            u32x4 t = q[0];
            opaque(t);
            held_offer<T, 1, TR>(hl, sp, q, v, in && held_vmax<T, TK_VALUES>(t) >= th, th, 0.0f);
        }
        n = 0;
        wave_sync();
    }
    __device__ __forceinline__ void end(HeldSmem<W>& sm, int wv, const HeldSpan<T>& sp, float ex) {
        const int tr = threadIdx.x;
        __syncthreads();  // (the maxima of the beginning have been read)
        const float t = word_value(team_bound<W, GRAN>(sm, order_word(lm), hl.K).lo);
        th = __builtin_fmaxf(th, t);
        if (n > 0) {
            keep();
            if (n > 0) look(sp);
        }
        hl.offer(tr < sp.ne && ex >= __builtin_fmaxf(th0, t),
                 make_key(ex, sp.base + (uint32_t)sp.extra(tr)));
        if (rare(hl.n > TH_CUT)) hl.cut();
        if ((tr & 63) == 0) sm.cnt[wv] = hl.n;
    }
};
struct NoPicks {};

template <typename T, bool SEL, bool ENT, int W>
__global__ __launch_bounds__(64 * W, 5) void logprob_stream(const LogprobRows a,
                                                            const LogprobSplit p) {
    constexpr int E = Vec<T>::N, TR = 64 * W, U = LS_U, OWN = SEL ? 1 : 0;
    __shared__ LogSmem<W, SEL> sm;
    __shared__ uint64_t notes[SEL ? W : 1][SEL ? TH_LIST : 1];
    const int tr = threadIdx.x, lane = tr & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tr >> 6);
    const uint32_t in_launch = blockIdx.x / (uint32_t)p.S;
    const int64_t row = p.row0 + in_launch;
    const int64_t start = (blockIdx.x - in_launch * (uint32_t)p.S) * p.chunk;
    const int64_t left = a.V - start;
    const T* xr = static_cast<const T*>(a.x) + row * a.ld;
    const HeldSpan<T> sp(xr, 0, start, 0, (int)(p.chunk < left ? p.chunk : left));
    const int nvec = sp.nvec;
    LogStream<T, ENT> st;
    st.c = a.c;
    // Steps of U vectors a lane, all whole but the last; of that, a lane loads the chunk's last
    // vector where it has none, and counts it as nothing.
    const int whole = nvec / (TR * U), steps = (nvec + TR * U - 1) / (TR * U);
    auto load = [&](u32x4 (&to)[U], int k) {
        if (k < whole) {
            const u32x4* const at = sp.vb + (int64_t)k * (TR * U);
#pragma unroll
            for (int u = 0; u < U; ++u) to[u] = __builtin_nontemporal_load(at + u * TR + tr);
        } else if (k < steps) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = tr + (k * U + u) * TR;
                to[u] = __builtin_nontemporal_load(sp.vb + (v < nvec ? v : nvec - 1));
            }
        }
    };
    std::conditional_t<SEL, LogPicks<T, W>, NoPicks> picks;
    auto step = [&](u32x4 (&q)[U], int k) {
        if (k == whole) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (tr + (k * U + u) * TR >= nvec) q[u] = st.nothing();
        }
        if constexpr (SEL) {
            const float v = st.step(q, picks.th);
            picks.step(sp, k, v);
        } else {
            st.step(q, __builtin_inff());
        }
    };
    LogToken tok;
    if (wv == OWN) tok.index(a, row, lane);
    u32x4 q0[U], q1[U];
    load(q0, 0);
    const float ex = tr < sp.ne ? load1(sp.xr + sp.extra(tr)) : -__builtin_inff();
    if (wv == OWN) tok.element(a, xr, lane);
    u32x4 extra = st.nothing();
    extra.x = E == 8 ? (0xFF800000u | __float_as_uint(ex) >> 16) : __float_as_uint(ex);
    if (sp.ne > 0) {
        u32x4 one[1] = {extra};
        st.step(one, __builtin_inff());
    }
    if constexpr (SEL) picks.begin(sm.top, notes[wv], wv, a.K, sp, q0, ex);
    for (int k = 0; k < steps; k += 2) {
        load(q1, k + 1);
        step(q0, k);
        if (k + 1 == steps) break;
        load(q0, k + 2);
        step(q1, k + 1);
    }
    LogState v;
    if (rare(st.far)) {  // again, one vector after the other
        v = log_of_vector<T>(extra, a.c);
        for (int i = tr; i < nvec; i += TR) v = log_merge(v, log_of_vector<T>(sp.vb[i], a.c), a.c);
        v = log_merge_wave(v, a.c);
    } else {
        v = st.end(ex, sp.vb, wv * 64, TR, nvec);
    }
    if constexpr (SEL) picks.end(sm.top, wv, sp, ex);
    if (lane == 0) sm.state[wv] = v;
    __syncthreads();
    if (p.S > 1) log_end<T, W, SEL, true>(a, p, sm, row, in_launch, blockIdx.x, tok);
    else log_end<T, W, SEL, false>(a, p, sm, row, in_launch, blockIdx.x, tok);
}

template <typename T, int W, bool SEL, bool ENT, bool PART>
hipError_t launch_logprob_w(const LogprobRows& a, const LogprobSplit& p, hipStream_t st) {
    const int64_t nv = (PART ? p.chunk : a.V) / Vec<T>::N;
    const int64_t r = (nv + 64 * W - 1) / (64 * W);
    const int64_t blocks = W == 1 ? (p.rows + TK_BLOCK / 64 - 1) / (TK_BLOCK / 64)
                                  : PART ? p.rows * p.S : p.rows;
    const dim3 grid((unsigned)blocks), block(W == 1 ? TK_BLOCK : 64 * W);
#define OSM_LOG(R_) \
    hipLaunchKernelGGL((logprob_held<T, W, R_, SEL, ENT, PART>), grid, block, 0, st, a, p)
    if constexpr (W == 1 && !SEL) {  // (shorter rows: launch_logprob_short)
        if (r <= 6) OSM_LOG(6);
        else if (r <= 8) OSM_LOG(8);
        else return hipErrorInvalidValue;
    } else if constexpr (W <= 4) {
        // (chunks have two vectors a lane and more)
        if (!PART && r <= 1) OSM_LOG((PART ? 2 : 1));
        else if (r <= 2) OSM_LOG(2);
        else if (r <= 4) OSM_LOG(4);
        else if (r <= 6) OSM_LOG(6);
        else if (r <= 8) OSM_LOG(8);
        else if constexpr (W == 4 && SEL) {
            if (r <= 12) OSM_LOG(12);
            else if (r <= TH_RMAX) OSM_LOG(16);
            else return hipErrorInvalidValue;
        } else {
            return hipErrorInvalidValue;
        }
    } else {
        if (r <= 8) OSM_LOG(8);
        else if (r <= 12) OSM_LOG(12);
        else if (r <= TH_RMAX) OSM_LOG(16);
        else return hipErrorInvalidValue;
    }
#undef OSM_LOG
    return hipGetLastError();
}

template <typename T, bool ENT>
hipError_t launch_logprob_short(const LogprobRows& a, const LogprobSplit& p, int lanes,
                                hipStream_t st) {
    const int64_t nv = a.V / Vec<T>::N, per = TK_BLOCK / lanes;
    const dim3 grid((unsigned)((p.rows + per - 1) / per)), block(TK_BLOCK);
#define OSM_SHORT(L, R_) \
    hipLaunchKernelGGL((logprob_short<T, ENT, L, R_>), grid, block, 0, st, a, p)
    if (lanes == 16) {
        if (nv <= 16) OSM_SHORT(16, 1);
        else if (nv <= 32) OSM_SHORT(16, 2);
        else if (nv <= 64) OSM_SHORT(16, 4);
        else return hipErrorInvalidValue;
    } else {
        if (nv <= 128) OSM_SHORT(32, 4);
        else if (nv <= 256) OSM_SHORT(32, 8);
        else return hipErrorInvalidValue;
    }
#undef OSM_SHORT
    return hipGetLastError();
}

template <typename T, bool SEL, bool ENT>
hipError_t launch_logprob_t(const LogprobRows& a, const LogprobPlan& plan, void* scratch,
                            uint32_t* ctr, hipStream_t st) {
    LogprobSplit p{};
    p.chunk = plan.chunk;
    p.S = plan.S;
    p.states = static_cast<uint64_t*>(scratch);
    p.keys = p.states + 2 * plan.rows * plan.S;
    p.ctr = ctr;
    for (p.row0 = 0; p.row0 < a.N; p.row0 += plan.rows) {
        p.rows = a.N - p.row0 < plan.rows ? a.N - p.row0 : plan.rows;
        hipError_t e;
        if (plan.stream) {
            const dim3 grid((unsigned)(p.rows * p.S));
            if constexpr (SEL) {
                hipLaunchKernelGGL((logprob_stream<T, SEL, ENT, 4>), grid, dim3(256), 0, st, a, p);
            } else {
                if (plan.stream == 8)
                    hipLaunchKernelGGL((logprob_stream<T, SEL, ENT, 8>), grid, dim3(512), 0, st, a,
                                       p);
                else
                    hipLaunchKernelGGL((logprob_stream<T, SEL, ENT, 4>), grid, dim3(256), 0, st, a,
                                       p);
            }
            e = hipGetLastError();
        } else if (plan.S > 1) {
            e = launch_logprob_w<T, 4, SEL, ENT, true>(a, p, st);
        } else if (plan.lanes) {
            if constexpr (SEL) e = hipErrorInvalidValue;
            else e = launch_logprob_short<T, ENT>(a, p, plan.lanes, st);
        } else if (plan.W == 1) {
            e = launch_logprob_w<T, 1, SEL, ENT, false>(a, p, st);
        } else if (plan.W == 4) {
            e = launch_logprob_w<T, 4, SEL, ENT, false>(a, p, st);
        } else {
            if constexpr (SEL) e = launch_logprob_w<T, 8, SEL, ENT, false>(a, p, st);
            else e = hipErrorInvalidValue;
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace osm
