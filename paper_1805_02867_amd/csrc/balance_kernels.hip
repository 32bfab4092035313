// The balance loss of a router's experts, with the counts and mean shares that it is made of,
// and its gradient.
//
// A row's shares are q = softmax(x), or the sigmoids over their sum; these are taken relative to
// the largest, e^{min(x, 0) - z} / (1 + e^-|x|) with z = max min(x, 0), so that they do not
// underflow together.  For a sequence of n rows (see balance_fwd)
//   loss = scale E / (K n^2) sum_e c_e sum_r q_re,
//   d loss / dx_rj = scale E / (K n^2) q_j (c_j - sum_e c_e q_e)      (times 1 - sigma_j).
// Balanced counts are all about K n / E and cancel in the gradient: they are taken less that
// number, which changes nothing as the shares sum to 1.
//
// Forward.  Workgroup b takes a span of rows; a row by a team of LANES lanes that hold R
// experts each, so that a lane sums the shares of its own experts over rows in registers (binary64:
// a sequence may be long), and counts go to LDS as integers, whose additions may come in any order.  At the end of each
// sequence's part of the span the teams' sums are joined in their order, in binary64.  A
// sequence that lies within the span is finished there.  Of others the parts go to scratch, and a
// second kernel joins them in the order of the spans, so that the result is the same every
// time.
//
// What bounds both is memory (a row is read once, the gradient written once), and for small
// batches the launches.
#include <type_traits>

#include "experts.hpp"
#include "kernels.h"

namespace osm {

constexpr int BL_BLOCK = 256;
constexpr int BL_WAVES = BL_BLOCK / 64;
constexpr int BL_JOIN = 1024;  // threads of the second kernel's workgroups
constexpr int BL_EMAX = 1024;

struct BalanceSpans {
    int64_t rows;    // of a span
    uint32_t spans;
    double* sums;    // spans * 2 * E: of the sequence before the span's first row, and of the last
    int32_t* counts; // the same
    int32_t* n;      // spans * 2
    int32_t* leads;  // the sequence that begins in the span and ends behind it, or -1
};

__device__ __forceinline__ int64_t seq_start(const BalanceRows& a, int64_t s) {
    if (!a.starts) return s == 0 ? 0 : a.N;
    const int64_t v = a.starts[s];
    return v < 0 ? 0 : v > a.N ? a.N : v;
}

// The first sequence that ends behind `row` (S: none), by the whole wavefront: 64 places at a
// time.
__device__ __forceinline__ int64_t seq_after(const BalanceRows& a, int64_t row) {
    if (!a.starts) return row < a.N ? 0 : 1;
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = a.S;  // the answer is in [lo, hi]
    while (hi > lo) {
        const int64_t step = (hi - lo + 63) / 64;
        const int64_t s = lo + lane * step;
        const bool behind = s < hi && seq_start(a, s + 1) > row;
        const uint64_t who = __ballot(behind);
        // the first of the places that does
        if (who == 0) {
            const int64_t last = lo + (hi - 1 - lo) / step * step;
            if (step == 1) return hi;
            lo = last + 1;
            continue;
        }
        const int f = __builtin_ctzll(who);
        hi = lo + f * step;
        lo = f == 0 ? hi : lo + (f - 1) * step + 1;
    }
    return lo;
}

// Shares of a row (see above), and for the gradient 1 - sigma of each expert.
template <int LANES, int R, bool SLOPE>
__device__ __forceinline__ void shares(const float (&x)[R], bool sigmoid, float (&q)[R],
                                       float (&slope)[R]) {
    float m = x[0];
    if (sigmoid) {
#pragma unroll
        for (int j = 1; j < R; ++j) m = fmaxf(m, x[j]);
        m = fminf(group_max<LANES>(m), 0.0f);
    } else {
#pragma unroll
        for (int j = 1; j < R; ++j) m = __builtin_elementwise_maximum(m, x[j]);
        m = team_maximum<LANES>(m);
    }
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        if (sigmoid) {
            const float e = exp2_hw(-__builtin_fabsf(x[j]) * kLog2e);
            const float f = __builtin_amdgcn_rcpf(1.0f + e);
            // (a NaN stays one: the minimum would give 0)
            const float z = x[j] > 0.0f ? 0.0f : x[j];
            q[j] = exp2_hw((z - m) * kLog2e) * f;
            if constexpr (SLOPE) slope[j] = x[j] > 0.0f ? e * f : f;
        } else {
            q[j] = exp2_hw((x[j] - m) * kLog2e);
            if constexpr (SLOPE) slope[j] = 1.0f;
        }
        sum += q[j];
    }
    const float r = 1.0f / group_sum<LANES>(sum);
#pragma unroll
    for (int j = 0; j < R; ++j) q[j] *= r;
}

// Whether one of a row's indices is an expert, for a team.  COUNT: they are counted.
template <int LANES, bool COUNT>
__device__ __forceinline__ bool takes_part(const BalanceRows& a, int64_t row, bool live, int lane,
                                           int team, int32_t* counts) {
    bool in = false;
    for (int k = lane; k < a.K; k += LANES) {
        const int32_t e = live ? a.idx[row * a.K + k] : -1;
        const bool is = e >= 0 && e < a.E;
        if (COUNT && is) atomicAdd(counts + e, 1);
        in = in || is;
    }
    const uint64_t who = __ballot(in);
    const uint64_t mine = LANES == 64 ? ~0ull : ((1ull << (LANES & 63)) - 1) << (team * LANES);
    return (who & mine) != 0;
}

// Loss, counts, mean shares and rows of sequence s by a workgroup, from sums[e] and counts[e]
// in LDS (or any memory that it may read after a barrier).
template <int THREADS>
__device__ __forceinline__ void finish(const BalanceRows& a, int64_t s, const double* sums,
                                       const int32_t* counts, int32_t n, double* part) {
    const double rn = n > 0 ? 1.0 / (double)n : 0.0;
    double dot = 0.0;
    for (int e = threadIdx.x; e < a.E; e += THREADS) {
        const double mean = sums[e] * rn;
        const int32_t c = counts[e];
        a.probs[s * a.E + e] = (float)mean;
        a.counts[s * a.E + e] = c;
        dot += (double)c * mean;
    }
    dot = group_sum<64>(dot);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int w = 0; w < THREADS / 64; ++w) all += part[w];
        a.loss[s] = (float)((double)a.scale * a.E / a.K * rn * all);
        a.rows[s] = n;
    }
}

template <typename T, int LANES, int R, int VEC>
__global__ __launch_bounds__(BL_BLOCK) void balance_spans(const BalanceRows a,
                                                          const BalanceSpans b) {
    constexpr int ROWS = 64 / LANES, TEAMS = BL_WAVES * ROWS;
    __shared__ double sums[LANES * R];
    __shared__ double acc[BL_WAVES][LANES * R];
    __shared__ int32_t counts[LANES * R];
    __shared__ int32_t part_rows[BL_WAVES];
    __shared__ double part[BL_WAVES];
    const int tid = threadIdx.x, lane = tid % LANES, wv = tid >> 6, team = (tid & 63) / LANES;
    const int E = a.E;
    const int64_t r0 = blockIdx.x * b.rows, r1 = r0 + b.rows < a.N ? r0 + b.rows : a.N;
    // its sequences: those that end behind r0 (all that end at row 0 are the first span's)
    int64_t s = blockIdx.x == 0 ? 0 : seq_after(a, r0);
    int32_t lead = -1;
    for (; s < a.S; ++s) {
        const int64_t from = seq_start(a, s), end = seq_start(a, s + 1);
        const int64_t to = end > from ? end : from;
        if (from > r1 || (from == r1 && to > from)) break;
        const int64_t p0 = from > r0 ? from : r0, p1 = to < r1 ? to : r1;
        for (int e = tid; e < LANES * R; e += BL_BLOCK) counts[e] = 0;
        __syncthreads();
        float q[R], none[R];
        double sum[R];
        int32_t n = 0;
#pragma unroll
        for (int j = 0; j < R; ++j) sum[j] = 0.0;
        for (int64_t row0 = p0 + wv * ROWS; row0 < p1; row0 += TEAMS) {
            const int64_t row = row0 + team;
            const bool live = row < p1;
            float x[R];
            load_experts<T, LANES, R, VEC>(static_cast<const T*>(a.x) + (live ? row : p0) * E, E,
                                           live, lane, x);
            const bool in = takes_part<LANES, true>(a, row, live, lane, team, counts);
            shares<LANES, R, false>(x, a.sigmoid, q, none);
#pragma unroll
            for (int j = 0; j < R; ++j) sum[j] += (double)(in ? q[j] : 0.0f);
            n += in && lane == 0;
        }
        // the wavefront's teams, then the wavefronts
#pragma unroll
        for (int d = LANES; d < 64; d *= 2) {
#pragma unroll
            for (int j = 0; j < R; ++j) sum[j] += __shfl_xor(sum[j], d);
        }
        if (team == 0) {
#pragma unroll
            for (int j = 0; j < R; ++j) acc[wv][expert<LANES, VEC>(lane, j)] = sum[j];
        }
        for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
        if ((tid & 63) == 0) part_rows[wv] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int w = 0; w < BL_WAVES; ++w) n += part_rows[w];
        const bool before = from < r0, behind = to > r1;
        const int slot = before ? 0 : 1;
        double* const out = before || behind ? b.sums + ((int64_t)blockIdx.x * 2 + slot) * E : sums;
        for (int e = tid; e < E; e += BL_BLOCK) {
            double v = 0.0;
#pragma unroll
            for (int w = 0; w < BL_WAVES; ++w) v += acc[w][e];
            out[e] = v;
        }
        if (before || behind) {
            int32_t* const oc = b.counts + ((int64_t)blockIdx.x * 2 + slot) * E;
            for (int e = tid; e < E; e += BL_BLOCK) oc[e] = counts[e];
            if (tid == 0) b.n[blockIdx.x * 2 + slot] = n;
            if (!before) lead = (int32_t)s;
        } else {
            __syncthreads();
            finish<BL_BLOCK>(a, s, sums, counts, n, part);
        }
        __syncthreads();
        if (behind) break;
    }
    if (tid == 0) b.leads[blockIdx.x] = lead;
}

// Sequences that more than one span has: workgroup i joins the one that begins in span i.
__global__ __launch_bounds__(BL_JOIN) void balance_join(const BalanceRows a,
                                                        const BalanceSpans b) {
    __shared__ double stripe[BL_JOIN];
    __shared__ int32_t stripe_counts[BL_JOIN];
    __shared__ double sums[BL_EMAX];
    __shared__ int32_t counts[BL_EMAX];
    __shared__ double part[BL_JOIN / 64];
    __shared__ int32_t rows[BL_JOIN / 64];
    const int64_t s = b.leads[blockIdx.x];
    if (s < 0) return;
    const int tid = threadIdx.x, E = a.E;
    const int64_t end = seq_start(a, s + 1);
    // slots: the second one of this span, the first ones of the following
    const int64_t i0 = blockIdx.x, more = (end - 1) / b.rows - i0;
    auto slot = [&](int64_t j) { return j == 0 ? i0 * 2 + 1 : (i0 + j) * 2; };
    const int cols = E < BL_JOIN ? E : BL_JOIN;
    const int stripes = BL_JOIN / cols, st = tid / cols, e = tid % cols;
    const int64_t each = (more + stripes) / stripes;  // slots of a stripe
    double v = 0.0;
    int32_t c = 0, n = 0;
    if (st < stripes) {
        const int64_t j1 = (st + 1) * each < more + 1 ? (st + 1) * each : more + 1;
#pragma unroll 8
        for (int64_t j = st * each; j < j1; ++j) {
            v += b.sums[slot(j) * E + e];
            c += b.counts[slot(j) * E + e];
        }
    }
    stripe[tid] = v;
    stripe_counts[tid] = c;
    for (int64_t j = tid; j <= more; j += BL_JOIN) n += b.n[slot(j)];
    for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
    if ((tid & 63) == 0) rows[tid >> 6] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < BL_JOIN / 64; ++w) n += rows[w];
    if (tid < cols) {
        v = 0.0;
        c = 0;
        for (int i = 0; i < stripes; ++i) {
            v += stripe[i * cols + tid];
            c += stripe_counts[i * cols + tid];
        }
        sums[tid] = v;
        counts[tid] = c;
    }
    __syncthreads();
    finish<BL_JOIN>(a, s, sums, counts, n, part);
}

template <typename T, int LANES, int R, int VEC>
__global__ __launch_bounds__(BL_BLOCK) void balance_grad(const BalanceRows a, int64_t span) {
    constexpr int ROWS = 64 / LANES, TEAMS = BL_WAVES * ROWS;
    const int tid = threadIdx.x, lane = tid % LANES, wv = tid >> 6, team = (tid & 63) / LANES;
    const int E = a.E;
    const int64_t r0 = blockIdx.x * span, r1 = r0 + span < a.N ? r0 + span : a.N;
    int64_t s = seq_after(a, r0 + wv * ROWS), s_end = -1, s_from = 0;  // of this lane's row
    float c[R], f = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) c[j] = 0.0f;
    for (int64_t row0 = r0 + wv * ROWS; row0 < r1; row0 += TEAMS) {
        const int64_t row = row0 + team;
        const bool live = row < r1;
        float x[R], q[R], slope[R];
        load_experts<T, LANES, R, VEC>(static_cast<const T*>(a.x) + (live ? row : r0) * E, E, live,
                                       lane, x);
        const bool in = takes_part<LANES, false>(a, row, live, lane, team, nullptr);
        if (live && row >= s_end) {  // another sequence
            while (s < a.S && (s_end = seq_start(a, s + 1)) <= row) ++s;
            if (s < a.S) {
                s_from = seq_start(a, s);
                const double n = (double)a.rows[s], mean = (double)a.K * n / E;
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const int e = expert<LANES, VEC>(lane, j);
                    c[j] = e < E ? (float)((double)a.counts[s * E + e] - mean) : 0.0f;
                }
                f = n > 0.0 ? (float)((double)a.dloss[s] * a.scale * E / (a.K * n * n)) : 0.0f;
            } else {
                s_from = s_end = INT64_MAX;  // behind the last
            }
        }
        const bool part = in && row >= s_from;
        shares<LANES, R, true>(x, a.sigmoid, q, slope);
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < R; ++j) dot = __builtin_fmaf(c[j], q[j], dot);
        dot = group_sum<LANES>(dot);
        if (!live) continue;
        T* dr = static_cast<T*>(a.dx) + row * E;
        float d[R];
#pragma unroll
        for (int j = 0; j < R; ++j) d[j] = part ? f * q[j] * (c[j] - dot) * slope[j] : 0.0f;
        store_experts<T, LANES, R, VEC>(dr, E, lane, d);
    }
}

// Lanes of a row: eight experts a lane or few more.
static int balance_lanes(int E) {
    int lanes = 8;
    while (lanes < 64 && lanes * 8 < E) lanes *= 2;
    return lanes;
}

// Rows of a span: as many as give every CU a workgroup or two, and at least four a team.
static int64_t balance_span(int64_t N, int E, int cus) {
    const int64_t teams = BL_BLOCK / balance_lanes(E);
    int64_t rows = (N + 2 * cus - 1) / (2 * (int64_t)cus);
    rows = (rows + teams - 1) / teams * teams;
    return rows < 4 * teams ? 4 * teams : rows;
}

static uint32_t balance_spans_of(int64_t N, int64_t rows) {
    return N > 0 ? (uint32_t)((N + rows - 1) / rows) : 1;
}

static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

size_t balance_scratch_bytes(int64_t N, int64_t E, int64_t S, int cus) {
    (void)S;
    const size_t spans = balance_spans_of(N, balance_span(N, (int)E, cus));
    return up256(spans * 2 * (size_t)E * 8) + up256(spans * 2 * (size_t)E * 4) +
           up256(spans * 2 * 4) + up256(spans * 4);
}

// Teams of LANES lanes with R experts each, VEC neighbours at a time: f is called with them as
// constants.
template <bool VEC4, typename F>
static void with_team(int E, F f) {
    constexpr int VEC = VEC4 ? 4 : 1;
    auto r = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const int each = (E + L - 1) / L;
        auto call = [&](auto n) { f(lanes, n, std::integral_constant<int, VEC>{}); };
        if constexpr (VEC == 1) {
            if (each <= 1) return call(std::integral_constant<int, 1>{});
            if (each <= 2) return call(std::integral_constant<int, 2>{});
        }
        if (each <= 4) return call(std::integral_constant<int, 4>{});
        if (L < 64 || each <= 8) return call(std::integral_constant<int, 8>{});
        if constexpr (L == 64) call(std::integral_constant<int, 16>{});
    };
    switch (balance_lanes(E)) {
        case 8: return r(std::integral_constant<int, 8>{});
        case 16: return r(std::integral_constant<int, 16>{});
        case 32: return r(std::integral_constant<int, 32>{});
        default: return r(std::integral_constant<int, 64>{});
    }
}

// Four neighbours at a time where every row allows it.
static bool four(const BalanceRows& a, size_t es, bool grad) {
    const uintptr_t at = (uintptr_t)a.x | (grad ? (uintptr_t)a.dx : 0);
    return a.E % 4 == 0 && a.E >= 32 && at % (4 * es) == 0;
}

template <typename T>
static hipError_t launch_balance_fwd_t(const BalanceRows& a, void* scratch, hipStream_t st) {
    BalanceSpans b{};
    b.rows = balance_span(a.N, a.E, a.cus);
    b.spans = balance_spans_of(a.N, b.rows);
    char* at = static_cast<char*>(scratch);
    b.sums = reinterpret_cast<double*>(at);
    at += up256((size_t)b.spans * 2 * a.E * 8);
    b.counts = reinterpret_cast<int32_t*>(at);
    at += up256((size_t)b.spans * 2 * a.E * 4);
    b.n = reinterpret_cast<int32_t*>(at);
    at += up256((size_t)b.spans * 2 * 4);
    b.leads = reinterpret_cast<int32_t*>(at);
    auto go = [&](auto lanes, auto r, auto vec) {
        hipLaunchKernelGGL((balance_spans<T, decltype(lanes)::value, decltype(r)::value,
                                          decltype(vec)::value>),
                           dim3(b.spans), dim3(BL_BLOCK), 0, st, a, b);
    };
    if (four(a, sizeof(T), false)) with_team<true>(a.E, go);
    else with_team<false>(a.E, go);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || b.spans == 1) return e;
    hipLaunchKernelGGL(balance_join, dim3(b.spans), dim3(BL_JOIN), 0, st, a, b);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_balance_bwd_t(const BalanceRows& a, hipStream_t st) {
    const int64_t teams = BL_BLOCK / balance_lanes(a.E);
    const int64_t want = (a.N + teams - 1) / teams, most = 8 * (int64_t)a.cus;
    const int64_t blocks = want < most ? want : most;
    const int64_t span = (a.N + blocks - 1) / blocks;
    auto go = [&](auto lanes, auto r, auto vec) {
        hipLaunchKernelGGL((balance_grad<T, decltype(lanes)::value, decltype(r)::value,
                                         decltype(vec)::value>),
                           dim3((unsigned)((a.N + span - 1) / span)), dim3(BL_BLOCK), 0, st, a,
                           span);
    };
    if (four(a, sizeof(T), true)) with_team<true>(a.E, go);
    else with_team<false>(a.E, go);
    return hipGetLastError();
}

hipError_t launch_balance_fwd(const BalanceRows& a, int dtype, void* scratch, hipStream_t st) {
    return dtype == 1 ? launch_balance_fwd_t<bf16_t>(a, scratch, st)
                      : launch_balance_fwd_t<float>(a, scratch, st);
}

hipError_t launch_balance_bwd(const BalanceRows& a, int dtype, hipStream_t st) {
    return dtype == 1 ? launch_balance_bwd_t<bf16_t>(a, st) : launch_balance_bwd_t<float>(a, st);
}

}  // namespace osm
