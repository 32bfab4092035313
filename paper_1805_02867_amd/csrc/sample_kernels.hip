// Kernels of softmax_sample (sample.hpp): rows held whole by a wavefront or a workgroup,
// rows split into chunks, and rows streamed from memory.
#include <type_traits>

#include "sample_values.hpp"

namespace osm {

constexpr int SM_W = 8;  // wavefronts of a workgroup that has a row, or a chunk, to itself
constexpr int SM_BLOCK = 64 * SM_W;

__device__ __forceinline__ void no_token(float* val, int32_t* idx) {
    *val = __builtin_nanf("");
    *idx = -1;
}

__device__ __forceinline__ SampleSmem<SM_W>& smem_of(ValueSmem& sm) { return sm.s; }
__device__ __forceinline__ SampleSmem<SM_W>& smem_of(SampleSmem<SM_W>& sm) { return sm; }
template <int W>
__device__ __forceinline__ SampleSmem<W>& smem_of(ListSmem<W>& sm) {
    return sm;
}

// bfloat16 rows of more than two vectors a lane of a workgroup go by their values, others by
// the bins of their weights: clearing and adding up 4096 bins takes shorter rows longer
// than it saves (1000 x 2000 top-p 63 us by values, 43 by weights; 1000 x 12000 84 and 109).
template <typename T, int W, int R>
using RowSmem =
    std::conditional_t<W == SM_W && R != 2 && std::is_same_v<T, bf16_t>, ValueSmem, ListSmem<W>>;
template <typename T, bool FILTERS>
using SplitSmem = std::conditional_t<
    FILTERS, std::conditional_t<std::is_same_v<T, bf16_t>, ValueSmem, ListSmem<SM_W>>,
    SampleSmem<SM_W>>;

// A row held by the team: loaded once.  False: it has to be done the slow way.
template <typename T, int W, int R>
__device__ __forceinline__ bool held_row(RowSmem<T, W, R>& rm, const T* x, int32_t V,
                                         const Rule& r, float* val, int32_t* idx) {
    constexpr bool VALUES = std::is_same_v<RowSmem<T, W, R>, ValueSmem>;
    SampleSmem<W>& sm = smem_of(rm);
    constexpr int THREADS = 64 * W, PER = SampleShape<W>::PER;
    const int tid = threadIdx.x % THREADS;
    [[maybe_unused]] const int lane = tid & 63;
    Held<T, W, R> h;
    h.load(x, V);
    const float m = team_maximum(sm, h.maximum());
    if (!(m < __builtin_inff()) || m == -__builtin_inff()) {
        if (tid == 0) no_token(val, idx);
        return true;
    }
    if (r.greedy) {
        const uint32_t at = index_of(sm, h, m);
        if (tid == 0) {
            *idx = (int32_t)at;
            *val = 1.0f;
        }
        return true;
    }
    const Anchor an = anchor(m, r.c);
    Cut cut = no_cut();
    if constexpr (VALUES) {
        if (r.k || r.p < 1.0) {
            clear_values(rm);
            __syncthreads();
            add_values(rm, h, an);
            __syncthreads();
            const ClassSum cl = {lane == 0 ? rm.mid : 0, lane == 0 ? rm.tail : 0,
                                 lane == 0 ? rm.mid_n : 0, lane == 0 ? rm.tail_n : 0};
            const double part = lane == 0 ? 1.0 : 0.0;
            const HeldCounts counts{rm.values};
            const Classes classes = in_row(cl, part);
            if (__builtin_expect(values_cut<false>(rm, r, an, 1, V, classes, part, h, counts,
                                                   [](int) {}, val, idx),
                                 1))
                return true;
            return values_lists<R>(rm, r, m, r.c, x, V, V, 1, classes, part, counts, val, idx);
        }
    } else if (r.k || r.p < 1.0) {
        if (cold((double)m * r.c)) return false;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            sm.mass[tid + j * THREADS] = 0;
            sm.counts[tid + j * THREADS] = 0;
        }
        team_sync<W>();
        bool tail = false;
        if (!r.k) add_histogram<true, false>(sm, h, an);
        else if (!(r.p < 1.0)) tail = add_histogram<false, true>(sm, h, an);
        else tail = add_histogram<true, true>(sm, h, an);
        tail = team_minimum(sm, tail ? 0u : 1u) == 0;
        team_sync<W>();
#pragma unroll
        for (int j = 0; j < PER; ++j)
            sm.sums[tid + j * THREADS] = (double)sm.mass[tid + j * THREADS] * 0x1p-48;
        team_sync<W>();
        const Filtered f = filter_row(rm, r, an, tail, (uint32_t)V - 1, false,
                                      [&](const Range& g) {
                                          h.each([&](const u32x4& v, int32_t i) {
                                              bool any = false;
#pragma unroll
                                              for (int e = 0; e < h.E; ++e)
                                                  any |= near(g, h.at(v, e));
                                              if (__ballot(any) == 0) return;
#pragma unroll
                                              for (int e = 0; e < h.E; ++e)
                                                  append(rm, g, an, h.at(v, e), (uint32_t)(i + e));
                                          });
                                      });
        if (!f.ok) return false;
        cut = f.cut;
    }
    return locate<false>(sm, h,
                  [&](const u32x4& v, uint32_t i, double(&w)[Vec<T>::N]) {
#pragma unroll
                      for (int e = 0; e < Vec<T>::N; ++e) {
                          w[e] = an.weight(h.at(v, e));
                          w[e] = cut.keeps(h.at(v, e), i + e) && w[e] >= r.q ? w[e] : 0.0;
                      }
                  },
                  r.u, 0.0, 0, val, idx);
}

// Short rows, a wavefront each.
constexpr int SM_SHORT = 1024;  // elements
template <typename T>
__global__ __launch_bounds__(256, 4) void sample_short(const SampleRows a) {
    constexpr int R = SM_SHORT / 64 / Vec<T>::N;
    __shared__ ListSmem<1> sm[4];
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t row = (int64_t)blockIdx.x * 4 + wv; row < a.N; row += (int64_t)gridDim.x * 4) {
        const T* x = static_cast<const T*>(a.x) + row * a.ld;
        const Rule r = row_rule(a, row);
        if (!held_row<T, 1, R>(sm[wv], x, (int32_t)a.V, r, a.vals + row, a.idx + row)) {
            wave_sync();
            sample_row(smem_of(sm[wv]), RowSource<T>{x, a.V}, r, a.vals + row, a.idx + row);
        }
        wave_sync();
    }
}

template <typename T, int R>
__global__ __launch_bounds__(SM_BLOCK, 4) void sample_rows(const SampleRows a) {
    __shared__ RowSmem<T, SM_W, R> sm;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.ld;
        const Rule r = row_rule(a, row);
        if (!held_row<T, SM_W, R>(sm, x, (int32_t)a.V, r, a.vals + row, a.idx + row)) {
            __syncthreads();
            sample_row(smem_of(sm), RowSource<T>{x, a.V}, r, a.vals + row, a.idx + row);
        }
        __syncthreads();
    }
}

template <typename T>
__global__ __launch_bounds__(SM_BLOCK) void sample_streamed(const SampleRows a) {
    __shared__ SampleSmem<SM_W> sm;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const RowSource<T> src{static_cast<const T*>(a.x) + row * a.ld, a.V};
        sample_row(sm, src, row_rule(a, row), a.vals + row, a.idx + row);
        __syncthreads();
    }
}

// ------------------------------------------------------------------ split rows
// What a chunk leaves for the workgroup that completes the row, at the device's
// coherence point: its maximum, the index of that (greedy rows) or whether elements
// of some weight lie below its histogram, and the sum of its weights relative to
// its own maximum (rows without a filter) or its histograms.
constexpr int SAMPLE_PART = 6;  // 64-bit words of a chunk: its sum, and its classes
static_assert(VB_BINS * 2 == SampleShape<SM_W>::BINS * 8, "counts take the place of masses");
struct ChunkSum {
    float m;
    uint32_t at;
    double z;
};

// The row's end, by the workgroup that put its last chunk.  False: the row has to be done
// the slow way.
template <typename T, int R, bool FILTERS>
__device__ __forceinline__ bool split_end(SplitSmem<T, FILTERS>& rm, const SampleRows& a,
                                          const SampleSplit& s, const T* x, const Rule& r,
                                          const uint64_t* parts, uint64_t* mass,
                                          const uint32_t* counts, float* val, int32_t* idx) {
    constexpr int BINS = SampleShape<SM_W>::BINS, PER = SampleShape<SM_W>::PER;
    constexpr int SUB = SampleShape<SM_W>::SUB, E = Vec<T>::N;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, S = s.S;
    constexpr bool VALUES = FILTERS && std::is_same_v<T, bf16_t>;
    SampleSmem<SM_W>& sm = smem_of(rm);
    // every wavefront: chunk `lane`
    float mc = -__builtin_inff();
    uint32_t at = 0;
    double z = 0.0;
    if (lane < S) {
        const uint64_t p0 = get(parts + SAMPLE_PART * lane);
        z = __builtin_bit_cast(double, get(parts + SAMPLE_PART * lane + 1));
        mc = __uint_as_float((uint32_t)p0);
        at = (uint32_t)(p0 >> 32);
    }
    const float m = wave_maximum(mc);
    if (!(m < __builtin_inff()) || m == -__builtin_inff()) {
        if (tid == 0) no_token(val, idx);
        return true;
    }
    if (r.greedy) {
        const int c = __builtin_ctzll(__ballot(mc == m));
        if (tid == c) {
            *idx = (int32_t)at;
            *val = 1.0f;
        }
        return true;
    }
    // a chunk far below the row's maximum has no weight at all
    const bool none = mc == -__builtin_inff() || ((double)mc - (double)m) * r.c < -1100.0;
    const bool filtered = FILTERS && (r.k || r.p < 1.0 || r.q > 0.0);
    const double part = none ? 0.0 : exp2_wide(((double)mc - (double)m) * r.c);
    if constexpr (VALUES) {
        if (filtered) {
            ClassSum cl = {0, 0, 0, 0};
            if (lane < S) {
                const uint64_t n = get(parts + SAMPLE_PART * lane + 4);
                cl = {get(parts + SAMPLE_PART * lane + 2), get(parts + SAMPLE_PART * lane + 3),
                      (uint32_t)n, (uint32_t)(n >> 32)};
            }
            const ScratchCounts counts{mass};
            const Anchor an = anchor(m, r.c);
            Classes classes = in_row(cl, part);
            if (!into_line(rm, an, classes, part, none ? 0 : value_base(m) - value_base(mc),
                           counts))
                return false;
            Held<T, SM_W, R> h;
            const RowParts<R> row{x, a.V, s.chunk};
            if (__builtin_expect(values_cut<false>(rm, r, an, S, s.chunk, classes, part, h, counts,
                                                   [&](int c) { row.hold(c, h); }, val, idx),
                                 1))
                return true;
            return values_lists<R>(rm, r, m, r.c, x, a.V, s.chunk, S, classes, part, counts, val,
                                   idx);
        }
    }
    // (the histograms leave out what is below 2^-64 of the largest weight; only a u at
    // the very ends of [0, 1] can fall there)
    const bool ends = r.u < 0x1p-30 || r.u > 1.0 - 0x1p-30;
    if (filtered && (__ballot(!none && cold((double)mc * r.c)) != 0 || ends)) return false;
    const Anchor an = anchor(m, r.c);
    // bins of the row's histogram that its own starts below, and its weights' factor
    const int down = none || !filtered ? 0 : (int)(an.a - anchor(mc, r.c).a) * SUB;
    Cut cut = no_cut();
    double kept = 0.0;  // of chunk `lane`
    if (!filtered) {
        kept = z * part;
    } else if constexpr (FILTERS && !VALUES) {
        // the row's histograms
        bool tail = r.k && __ballot(lane < S && !none && at != 0) != 0;
        double sum[PER];
        uint32_t num[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            sum[j] = 0.0;
            num[j] = 0;
        }
        constexpr int AT_ONCE = 4;  // chunks whose loads are in flight
        for (int c0 = 0; c0 < S; c0 += AT_ONCE) {
            uint64_t w[AT_ONCE][PER];
            uint32_t n[AT_ONCE][PER];
            int off[AT_ONCE];
            double part_c[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int c = c0 + k < S ? c0 + k : S - 1;
                off[k] = __builtin_amdgcn_readlane(down, c);
                part_c[k] = c0 + k < S ? lane_value(part, c) : 0.0;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int b = tid + j * SM_BLOCK - off[k];
                    const bool in = b >= 0 && part_c[k] > 0.0;
                    w[k][j] = in ? get(mass + (int64_t)c * BINS + b) : 0;
                    n[k][j] = in && r.k ? get(counts + (int64_t)c * BINS + b) : 0;
                }
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    sum[j] += (double)w[k][j] * 0x1p-48 * part_c[k];
                    num[j] += n[k][j];
                }
                // what a shift moves out of the window
                if (r.k && part_c[k] > 0.0)
                    for (int b = BINS - 1 - off[k] + tid; b < BINS; b += SM_BLOCK)
                        tail |= b >= 0 && get(counts + (int64_t)(c0 + k) * BINS + b) != 0;
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int b = tid + j * SM_BLOCK;
            sm.sums[b] = b < BINS - 1 ? sum[j] : 0.0;
            sm.counts[b] = b < BINS - 1 ? num[j] : 0;
        }
        tail = team_minimum(sm, tail ? 0u : 1u) == 0;
        __syncthreads();
        const Filtered f = filter_row(
            rm, r, an, tail, (uint32_t)a.V - 1, true, [&](const Range& g) {
                const int h = (int)(((uintptr_t)x & 15) / sizeof(T));
                const int64_t vecs = (a.V + h + E - 1) / E;
                constexpr int AT_ONCE = 8;
                for (int64_t v0 = 0; v0 < vecs; v0 += AT_ONCE * SM_BLOCK) {
                    u32x4 q[AT_ONCE];
                    int64_t i0 = (v0 + tid) * E - h;
#pragma unroll
                    for (int j = 0; j < AT_ONCE; ++j) {
                        const int64_t i = i0 + j * SM_BLOCK * E;
                        if (i >= 0 && i + E <= a.V) q[j] = *reinterpret_cast<const u32x4*>(x + i);
                    }
#pragma unroll 1
                    for (int j = 0; j < AT_ONCE; ++j) {
                        const bool whole = i0 >= 0 && i0 + E <= a.V;
                        float v[E];
                        bool any = false;
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const int64_t i = i0 + e;
                            v[e] = whole                ? elem(q[0], e, (T*)nullptr)
                                   : i >= 0 && i < a.V ? load1(x + i)
                                                       : -__builtin_inff();
                            any |= near(g, v[e]);
                        }
                        if (__ballot(any) != 0) {
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                append(rm, g, an, v[e], (uint32_t)(i0 + e));
                        }
#pragma unroll
                        for (int k = 0; k + 1 < AT_ONCE; ++k) q[k] = q[k + 1];
                        i0 += SM_BLOCK * E;
                    }
                }
            });
        if (!f.ok) return false;
        cut = f.cut;
        // the kept weights of each chunk: of the bins kept whole, and of the list
        const int n = f.sure < BINS - 1 ? sm.n : 0;
        if (tid < 64) sm.chunk[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += SM_BLOCK) {
            const float v = rm.lx[j];
            const uint32_t i = rm.li[j];
            const double w = an.weight(v);
            if (an.bin<SM_W>(an.t(v)) >= f.sure && cut.keeps(v, i) && w >= r.q)
                add_bin(sm.chunk[i / (uint32_t)s.chunk], fixed48(w));
        }
        __syncthreads();
        kept = (double)sm.chunk[lane] * 0x1p-48;
        for (int c = wv; c < S; c += SM_W) {
            const int off = __builtin_amdgcn_readlane(down, c);
            const double part_c = lane_value(part, c);
            uint64_t units = 0;
            if (part_c > 0.0)
                for (int b = lane; b + off < f.sure; b += 64)
                    units += get(mass + (int64_t)c * BINS + b);
            units = wave_total(units);
            if (lane == 0) sm.whole[c] = (double)units * 0x1p-48 * part_c;
        }
        __syncthreads();
        kept += lane < S ? sm.whole[lane] : 0.0;
    }
    // the chunk that the token is in (every wavefront: the same numbers)
    const double incl = wave_scan(kept);
    const double total = lane_value(incl, 63), target = r.u * total;
    const uint64_t some = __ballot(kept > 0.0), past = __ballot(kept > 0.0 && incl > target);
    const int c = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : 0;
    const double rem = past ? target - (c ? lane_value(incl, c - 1) : 0.0) : __builtin_inf();
    const int64_t i0 = (int64_t)c * s.chunk;
    Held<T, SM_W, R> h;
    h.load(x + i0, (int32_t)(a.V - i0 < s.chunk ? a.V - i0 : s.chunk));
    __syncthreads();
    return locate<true>(sm, h,
                        [&](const u32x4& v, uint32_t i, double(&w)[E]) {
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                w[e] = an.weight(h.at(v, e));
                                const bool in = cut.keeps(h.at(v, e), (uint32_t)i0 + i + e);
                                w[e] = in && w[e] >= r.q ? w[e] : 0.0;
                            }
                        },
                        rem, total, (uint32_t)i0, val, idx);
}

// A chunk of a row a workgroup.  Workgroups go to the eight dies in turn, and there to
// groups of CUs in turn, each waiting for room where its turn is; and the one that
// ends a row is as a rule the last of its chunks to start.  With a row's chunks side by
// side every row ends at the same few places, for which the next ones then wait.  So the
// chunks of 32 rows are interleaved: rows end at 32 places in turn, and a row's chunks are
// on one die, whose L2 has their sums (side by side and interleaved: 512 x 128256 bfloat16
// top-p, eight chunks a row, 234 and 100 us; 256 x 128256 binary32 without filters 75 and
// 47).  Fewer than eight rows spread theirs over all dies.
// Without FILTERS every row draws from its whole distribution (or takes its maximum).
template <typename T, int R, bool FILTERS>
__global__ __launch_bounds__(SM_BLOCK, FILTERS ? 4 : 6) void sample_split(const SampleRows a,
                                                                         const SampleSplit s) {
    constexpr int BINS = SampleShape<SM_W>::BINS, PER = SampleShape<SM_W>::PER;
    __shared__ SplitSmem<T, FILTERS> rm;
    SampleSmem<SM_W>& sm = smem_of(rm);
    const int tid = threadIdx.x;
    const unsigned S = (unsigned)s.S, b = blockIdx.x, group = (unsigned)s.group;
    const int64_t rel = (int64_t)(b / (group * S) * group + b % group);
    const int c = (int)(b / group % S);
    if (rel >= s.rows) return;
    const int64_t row = s.row0 + rel;
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    const Rule r = row_rule(a, row);
    uint64_t* parts = s.parts + rel * s.S * SAMPLE_PART;
    uint64_t* mass = s.mass + rel * s.S * BINS;
    uint32_t* counts = s.counts + rel * s.S * BINS;
    {
        const int64_t i0 = (int64_t)c * s.chunk;
        Held<T, SM_W, R> h;
        h.load(x + i0, (int32_t)(a.V - i0 < s.chunk ? a.V - i0 : s.chunk));
        ChunkSum p{team_maximum(sm, h.maximum()), 0, 0.0};
        const bool live = p.m < __builtin_inff() && p.m > -__builtin_inff();
        if (r.greedy) {
            p.at = index_of(sm, h, p.m) + (uint32_t)i0;
        } else if (live) {
            const Anchor an = anchor(p.m, r.c);
            if (!FILTERS || !(r.k || r.p < 1.0 || r.q > 0.0)) {
                p.z = sum_weights(sm, h, an);
            } else if constexpr (!FILTERS) {
            } else if constexpr (std::is_same_v<T, bf16_t>) {
                clear_values(rm);
                __syncthreads();
                add_values(rm, h, an);
                __syncthreads();
                // 16 bits a bin: a chunk has at most 2^15 elements
                const uint32_t* v = rm.values + VB_PER * tid;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    put(mass + (int64_t)c * BINS + 2 * tid + j,
                        (uint64_t)(v[4 * j + 2] | v[4 * j + 3] << 16) << 32 |
                            (v[4 * j] | v[4 * j + 1] << 16));
                if (tid == 0) {
                    put(parts + SAMPLE_PART * c + 2, rm.mid);
                    put(parts + SAMPLE_PART * c + 3, rm.tail);
                    put(parts + SAMPLE_PART * c + 4, (uint64_t)rm.tail_n << 32 | rm.mid_n);
                }
            } else if (!cold((double)p.m * r.c)) {
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    sm.mass[tid + j * SM_BLOCK] = 0;
                    sm.counts[tid + j * SM_BLOCK] = 0;
                }
                __syncthreads();
                bool tail = false;
                if (!r.k) add_histogram<true, false>(sm, h, an);
                else tail = add_histogram<true, true>(sm, h, an);
                p.at = team_minimum(sm, tail ? 0u : 1u) == 0;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int b = tid + j * SM_BLOCK;
                    put(mass + (int64_t)c * BINS + b, sm.mass[b]);
                    if (r.k) put(counts + (int64_t)c * BINS + b, sm.counts[b]);
                }
            }
        }
        if (tid == 0) {
            put(parts + SAMPLE_PART * c, (uint64_t)p.at << 32 | __float_as_uint(p.m));
            put(parts + SAMPLE_PART * c + 1, __builtin_bit_cast(uint64_t, p.z));
        }
    }
    // every store of the chunk has completed before the row's count moves
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0)
        sm.found = (int)__hip_atomic_fetch_add(s.ctr + rel, 1u, __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const int done = sm.found;
    __syncthreads();
    if (done != s.S - 1) return;
    if (tid == 0) __hip_atomic_store(s.ctr + rel, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool ok =
        split_end<T, R, FILTERS>(rm, a, s, x, r, parts, mass, counts, a.vals + row, a.idx + row);
    if constexpr (FILTERS) {  // (without filters the histograms have nothing to decide)
        if (ok) return;
        __syncthreads();
        sample_row(sm, RowSource<T>{x, a.V}, r, a.vals + row, a.idx + row);
    }
}

// ------------------------------------------------------------------------ plan
namespace {
constexpr int kSplitMax = 64;            // chunks of a row: a lane each
constexpr int64_t kSplitChunks = 4096;   // of one launch, which bounds the scratch

template <typename T>
constexpr int64_t held_elems(int R) {
    return (int64_t)SM_BLOCK * R * Vec<T>::N;
}
}  // namespace

bool sample_filters(const SampleRows& a) {
    return a.top_k || a.top_p || a.min_p || (a.top_k_all > 0 && a.top_k_all < a.V) ||
           a.top_p_all < 1.0f || a.min_p_all > 0.0f;
}

SamplePlan sample_plan(int64_t N, int64_t V, int64_t ld, bool aligned, int dtype, bool filters,
                       int cus) {
    const int E = dtype == 1 ? 8 : 4;
    const int64_t room = V + (aligned && ld % E == 0 ? 0 : E - 1);
    const int64_t one = (int64_t)SM_BLOCK * E;  // a vector a lane
    if (room <= SM_SHORT) return {0, 1, V, 1};
    if (room <= 2 * one) return {2, 1, V, 1};
    // Chunks of whole vectors, at most four a lane: with eight the kernels without filters
    // take so many registers that fewer workgroups fit on a CU (256 x 128256 binary32 59 us,
    // with four 47); eight where a row would have too many chunks.  Fewer rows than fill the
    // chip are split further, into up to four chunks, whose sums the row's end has in flight
    // at once (60 x 16000 binary32 top-p: 32.2 us with four, 33.5 with the two that it needs,
    // 37.0 with seven).
    // Binary32 rows with filters take eight as well where that saves a launch (which waits for
    // the one before) or, of more than four chunks, half a launch's: their histograms are what a
    // row's end reads, and their kernels have the registers (top-p, us with eight and four:
    // 128 x 128256 102 and 95, 250 x 128256 126 and 133, 300 x 128256 138 and 216; 1000 x 20000
    // 134 and 121, 1400 x 20000 174 and 193, 2100 x 20000 282 and 252).
    const auto chunks = [&](int64_t r) { return (V + r * one - E - 1) / (r * one - E); };
    const auto launches = [&](int64_t s) {
        const int64_t rows = kSplitChunks / s;
        return (N + rows - 1) / rows;
    };
    int64_t R = 4, least = chunks(4);
    const int64_t eight = chunks(8);
    if (least > kSplitMax ||
        (filters && dtype != 1 && eight > 1 &&
         ((least > 4 && N * least > kSplitChunks / 2) || launches(eight) < launches(least)))) {
        R = 8;
        least = eight;
    }
    int64_t S = 2 * (int64_t)cus / (N > 0 ? N : 1);
    const int64_t most = V / one;
    S = S < 4 ? S : 4;
    S = S < most ? S : most;
    S = S > least ? S : least;
    if (S > kSplitMax) return {-1, 1, V, 1};
    if (S <= 1) return {4, 1, V, 1};
    int64_t chunk = (V + S - 1) / S;
    chunk = (chunk + E - 1) / E * E;
    S = (V + chunk - 1) / chunk;
    R = chunk + E <= 2 * one ? 2 : R;
    int64_t rows = kSplitChunks / S;
    rows = rows < N ? rows : N;
    return {(int)R, (int)S, chunk, rows > 0 ? rows : 1};
}

size_t sample_scratch_bytes(const SamplePlan& p) {
    if (p.S <= 1) return 0;
    constexpr size_t BINS = SampleShape<SM_W>::BINS;
    return (size_t)p.rows * (size_t)p.S * (8 * SAMPLE_PART + 12 * BINS);
}

template <typename T>
static hipError_t launch_sample_t(const SampleRows& a, const SamplePlan& p, void* scratch,
                                  uint32_t* ctr, hipStream_t st) {
    // (a launch takes fewer than 2^32 threads: further rows by the same workgroups)
    const auto blocks = [](int64_t n) { return dim3((unsigned)(n < (1 << 22) ? n : 1 << 22)); };
    if (p.S <= 1) {
        if (p.R == 0)
            hipLaunchKernelGGL(sample_short<T>, blocks((a.N + 3) / 4), dim3(256), 0, st, a);
        else if (p.R == 2)
            hipLaunchKernelGGL((sample_rows<T, 2>), blocks(a.N), dim3(SM_BLOCK), 0, st, a);
        else if (p.R > 0)
            hipLaunchKernelGGL((sample_rows<T, 4>), blocks(a.N), dim3(SM_BLOCK), 0, st, a);
        else
            hipLaunchKernelGGL(sample_streamed<T>, blocks(a.N), dim3(SM_BLOCK), 0, st, a);
        return hipGetLastError();
    }
    constexpr int64_t BINS = SampleShape<SM_W>::BINS;
    const bool filters = sample_filters(a);
    SampleSplit s;
    s.S = p.S;
    s.chunk = p.chunk;
    s.parts = static_cast<uint64_t*>(scratch);
    s.mass = s.parts + p.rows * p.S * SAMPLE_PART;
    s.counts = reinterpret_cast<uint32_t*>(s.mass + p.rows * p.S * BINS);
    s.ctr = ctr;
    for (s.row0 = 0; s.row0 < a.N; s.row0 += p.rows) {
        const int64_t n = a.N - s.row0 < p.rows ? a.N - s.row0 : p.rows;
        s.rows = n;
        s.group = n < 8 ? 1 : n < 32 ? 8 : 32;
        const dim3 grid((unsigned)((n + s.group - 1) / s.group * s.group * p.S)), block(SM_BLOCK);
        const auto launch = [&](auto filters) {
            constexpr bool F = decltype(filters)::value;
            const auto kernel = p.R == 2   ? sample_split<T, 2, F>
                                : p.R == 4 ? sample_split<T, 4, F>
                                           : sample_split<T, 8, F>;
            hipLaunchKernelGGL(kernel, grid, block, 0, st, a, s);
        };
        if (filters) launch(std::true_type{});
        else launch(std::false_type{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_sample(const SampleRows& a, const SamplePlan& p, int dtype, void* scratch,
                         uint32_t* ctr, hipStream_t st) {
    return dtype == 1 ? launch_sample_t<bf16_t>(a, p, scratch, ctr, st)
                      : launch_sample_t<float>(a, p, scratch, ctr, st);
}

}  // namespace osm
