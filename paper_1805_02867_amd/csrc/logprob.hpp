// Log probabilities of given tokens, the entropy and the best alternatives of rows (or chunks
// of rows) held in registers: one read of every element.
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
// Exponents are formed as (x - m) c, not as one fma with m c: the difference is exact near the
// maximum at any magnitude of the logits, and the largest element's exponent is 0.
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
    return {hi.m, __builtin_fmaf(d, r, hi.s), __builtin_fmaf(__builtin_fmaf(fall, d, lo.w), r, hi.w)};
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

// Adds a vector's weights and falls.  skip: an element of value m is left out, the first.
template <bool SKIP, int E>
__device__ __forceinline__ void log_add(const float (&x)[E], float m, float c, float& s, float& w) {
    bool done = !SKIP;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float t = (x[e] - m) * c;
        float p = exp2_hw(t);
        if constexpr (SKIP) {
            const bool is = !done && x[e] == m;
            p = is ? 0.0f : p;
            done = done || is;
        }
        s += p;
        w = __builtin_fmaf(p, -__builtin_fmaxf(t, kLogFloor), w);
    }
}

// What lane l < T of a wavefront knows of its row's l-th token.
struct LogToken {
    float x;
    bool in;
};

template <typename T>
__device__ __forceinline__ LogToken log_token(const LogprobRows& a, const T* xr, int64_t row,
                                              int lane) {
    LogToken t{0.0f, false};
    if (lane < a.T) {
        const int32_t i = a.tokens[row * a.T + lane];
        t.in = i >= 0 && (int64_t)i < a.V;
        if (t.in) t.x = load1(xr + i);
    }
    return t;
}

// A row's outputs by one wavefront, from its state, lane l's token and (SEL) l-th key.
template <bool SEL>
__device__ __forceinline__ void log_store(const LogprobRows& a, int64_t row, LogState v,
                                          LogToken t, uint64_t key) {
    const int lane = threadIdx.x & 63;
    const bool good = __builtin_fabsf(v.m) < __builtin_inff() && v.s == v.s;
    const float nan = __builtin_nanf("");
    const double s = (double)v.s, ln_d = log1p(s), m = (double)v.m;
    if (lane < a.T) {
        const float lp = (float)(((double)t.x - m) * a.inverse - ln_d);
        a.logp[row * a.T + lane] = !t.in ? 0.0f : good ? lp : nan;
    }
    if (lane == 0) {
        if (a.entropy) {
            const double h = ln_d + 0.69314718055994530942 * (double)v.w / (1.0 + s);
            a.entropy[row] = good ? (float)h : nan;
        }
        if (a.stats) {
            a.stats[row * 2] = good ? v.m : nan;
            a.stats[row * 2 + 1] = good ? v.s : nan;
        }
    }
    if constexpr (SEL) {
        if (lane < a.K) {
            const float lp = (float)(((double)key_value(key) - m) * a.inverse - ln_d);
            a.top_vals[row * a.K + lane] = good ? lp : nan;
            a.top_idx[row * a.K + lane] = good ? key_index(key) : -1;
        }
    }
}

// LDS of a workgroup.
template <int W, bool SEL>
struct LogSmem {
    LogState state[W];
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

// Rows (PART = false) or chunks of rows (PART = true: workgroup b has chunk b % S of row
// row0 + b / S) of at most 64 W R whole 16-byte vectors, W wavefronts each (W = 1: four rows a
// workgroup).  SEL: with alternatives, selected as topk_held.hpp does.
template <typename T, int W, int R, bool SEL, bool PART>
__global__ __launch_bounds__(W == 1 ? TK_BLOCK : 64 * W, (held_waves<T, W, R, PART>())) void logprob_held(
    const LogprobRows a, const LogprobSplit p) {
    static_assert(!PART || W > 1, "chunks take a workgroup each");
    constexpr int E = Vec<T>::N, TR = 64 * W;
    constexpr uint32_t GRAN = E == 8 ? 1u << 16 : 1u;
    __shared__ LogSmem<W, SEL> sm;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tr = W == 1 ? lane : tid;
    const int64_t vr = W == 1 ? (int64_t)blockIdx.x * (TK_BLOCK / 64) + wv : (int64_t)blockIdx.x;
    if (W == 1 && vr >= a.N) return;  // whole wavefronts; no barrier follows
    const uint32_t in_launch = PART ? blockIdx.x / (uint32_t)p.S : 0;
    const int64_t row = PART ? p.row0 + in_launch : vr;
    const int64_t start = PART ? (blockIdx.x - in_launch * (uint32_t)p.S) * p.chunk : 0;
    const int64_t left = a.V - start;
    const T* xr = static_cast<const T*>(a.x) + row * a.ld;
    const HeldSpan<T> sp(xr, 0, start, 0, (int)(PART && p.chunk < left ? p.chunk : left));
    const int nvec = sp.nvec;
    const float ninf = -__builtin_inff(), c = a.c;

    // all loads first; lanes past the row load its last vector and mask it
    u32x4 buf[R];
    if (nvec > 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int v = tr + i * TR;
            buf[i] = __builtin_nontemporal_load(sp.vb + (v < nvec ? v : nvec - 1));
        }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) buf[i] = u32x4{0, 0, 0, 0};
    }
    const float ex = tr < sp.ne ? load1(sp.xr + sp.extra(tr)) : ninf;
    LogToken tok{0.0f, false};
    if (wv == 0 || W == 1) tok = log_token(a, xr, row, lane);

    // 1. maxima by vector, and the wavefront's
    float vm[R];
    float lm = __builtin_fmaxf(ex, ninf);  // a NaN element gives -inf
#pragma unroll
    for (int i = 0; i < R; ++i) {
        vm[i] = tr + i * TR < nvec ? held_vmax<T, TK_VALUES>(buf[i]) : ninf;
        lm = max3_raw(lm, vm[i], ninf);
    }
    const float wm = wave_max_f(lm);
    // 2. the wavefront's state.  The element that is left out: the head or tail element of
    // the first lane that has the maximum there, else in that lane's vector `left_out`, which is
    // looked at again by itself.
    LogState st;
    {
        const float m = wm > ninf ? wm : 0.0f;  // (no elements, or only -inf)
        float s = 0.0f, w = 0.0f;
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
        {
            const float x1[1] = {ex};
            if (!(mine && at_ex != 0)) log_add<false>(x1, m, c, s, w);
        }
        u32x4 again = buf[0];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            opaque(buf[i]);
            if (i == 0 || i * TR < nvec) {  // uniform
                float xv[E], ps = 0.0f, pw = 0.0f;
                widen<T>(buf[i], xv);
                log_add<false>(xv, m, c, ps, pw);
                bool counts = tr + i * TR < nvec;
                if (i == left_out) {  // uniform
                    again = buf[i];
                    counts = counts && !mine;
                }
                s += counts ? ps : 0.0f;
                w += counts ? pw : 0.0f;
            }
        }
        if (left_out >= 0) {
            float xv[E], ps = 0.0f, pw = 0.0f;
            widen<T>(again, xv);
            log_add<true>(xv, m, c, ps, pw);
            s += mine ? ps : 0.0f;
            w += mine ? pw : 0.0f;
        }
        s = group_sum<64>(s);
        w = group_sum<64>(w);
        st = LogState{wm, wm > ninf ? s : s - 1.0f, w};
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
        log_store<SEL>(a, row, st, tok, key);
    } else {
        if (lane == 0) sm.state[wv] = st;
        __syncthreads();
        bool last = false;
        if (wv == 0) {
            st = sm.state[0];
#pragma unroll
            for (int i = 1; i < W; ++i) st = log_merge(st, sm.state[i], c);
            if constexpr (SEL) key = held_finish<W>(sm.top.list, sm.top.cnt, a.K);
            if constexpr (!PART) {
                log_store<SEL>(a, row, st, tok, key);
            } else {
                // the partial, at the device's coherence point; then the row's count
                if (SEL && lane < a.K)
                    __hip_atomic_store(p.keys + vr * a.K + lane, key, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
                if (lane == 0) log_put(p.states + vr * 2, st);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                uint32_t done = 0;
                if (lane == 0)
                    done = __hip_atomic_fetch_add(p.ctr + in_launch, 1u, __ATOMIC_RELAXED,
                                                  __HIP_MEMORY_SCOPE_AGENT);
                last = __builtin_amdgcn_readfirstlane(done) == (uint32_t)p.S - 1;
            }
        }
        if constexpr (PART) {
            const int64_t first = (int64_t)in_launch * p.S;  // the row's first chunk
            if constexpr (!SEL) {
                if (!last) return;
                // every chunk of the row is in
            } else {
                // a merge of more partial keys than one wavefront holds takes them all
                const bool wide = (int64_t)p.S * a.K > 64 * TK_MERGE_B;
                if (wide) {
                    if (wv == 0 && lane == 0) sm.top.cnt[0] = last;
                    __syncthreads();
                    last = sm.top.cnt[0] != 0;
                    __syncthreads();
                }
                if (!last) return;
                const uint64_t* pk = p.keys + first * a.K;
                const int64_t n = (int64_t)p.S * a.K;
                MD none;
                if (wide) {
                    if (!held_merge<TK_VALUES, W, TK_MERGE_B, GRAN, true>(sm.top, wv, pk, nullptr,
                                                                         n, 0, a.K, &key, &none))
                        return;
                } else {
                    held_merge<TK_VALUES, 1, TK_MERGE_B, GRAN, true>(sm.top, 0, pk, nullptr, n, 0,
                                                                    a.K, &key, &none);
                }
            }
            LogState v = log_empty();
            for (int j = lane; j < p.S; j += 64)
                v = log_merge(v, log_get(p.states + (first + j) * 2), c);
            log_store<SEL>(a, row, log_merge_wave(v, c), tok, key);
            if (lane == 0)
                __hip_atomic_store(p.ctr + in_launch, 0u, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
    }
}

template <typename T, int W, bool SEL, bool PART>
hipError_t launch_logprob_w(const LogprobRows& a, const LogprobSplit& p, hipStream_t st) {
    const int64_t nv = (PART ? p.chunk : a.V) / Vec<T>::N;
    const int64_t r = (nv + 64 * W - 1) / (64 * W);
    const int64_t blocks = W == 1 ? (a.N + TK_BLOCK / 64 - 1) / (TK_BLOCK / 64)
                                  : PART ? p.rows * p.S : a.N;
    const dim3 grid((unsigned)blocks), block(W == 1 ? TK_BLOCK : 64 * W);
#define OSM_LOG(R_) \
    hipLaunchKernelGGL((logprob_held<T, W, R_, SEL, PART>), grid, block, 0, st, a, p)
    if constexpr (W <= 4) {
        if (r <= 1) OSM_LOG(1);
        else if (r <= 2) OSM_LOG(2);
        else if (r <= 4) OSM_LOG(4);
        else if (r <= 6) OSM_LOG(6);
        else if (r <= 8) OSM_LOG(8);
        else if (r <= 12) OSM_LOG(12);
        else if (r <= TH_RMAX) OSM_LOG(16);
        else return hipErrorInvalidValue;
    } else {
        if (r <= 8) OSM_LOG(8);
        else if (r <= 12) OSM_LOG(12);
        else if (r <= TH_RMAX) OSM_LOG(16);
        else return hipErrorInvalidValue;
    }
#undef OSM_LOG
    return hipGetLastError();
}

template <typename T, bool SEL>
hipError_t launch_logprob_t(const LogprobRows& a, const LogprobPlan& plan, void* scratch,
                            uint32_t* ctr, hipStream_t st) {
    LogprobSplit p{};
    p.chunk = plan.chunk;
    p.S = plan.S;
    if (plan.S <= 1) {
        switch (plan.W) {
            case 1: return launch_logprob_w<T, 1, SEL, false>(a, p, st);
            case 4: return launch_logprob_w<T, 4, SEL, false>(a, p, st);
            case 8: return launch_logprob_w<T, 8, SEL, false>(a, p, st);
            default: return hipErrorInvalidValue;
        }
    }
    p.states = static_cast<uint64_t*>(scratch);
    p.keys = p.states + 2 * plan.rows * plan.S;
    p.ctr = ctr;
    for (p.row0 = 0; p.row0 < a.N; p.row0 += plan.rows) {
        p.rows = a.N - p.row0 < plan.rows ? a.N - p.row0 : plan.rows;
        const hipError_t e = plan.W == 4 ? launch_logprob_w<T, 4, SEL, true>(a, p, st)
                                         : launch_logprob_w<T, 8, SEL, true>(a, p, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace osm
