// The balance loss of a router's experts, with the counts and mean shares that it is made of,
// and its gradient.
//
// A row's shares are q = softmax(x), or the sigmoids 1 / (1 + e^-x) over their sum.  Where that sum
// is below 2^-60, all x are far below 0 and the sigmoids e^x but for 2^-60 of them: there they
// are e^{x - max x}, which does not underflow.  In other rows a sigmoid below 2^-126 is 0, a
// share of less than 2^-66.  For a sequence of n rows (see balance_fwd)
//   loss = scale E / (K n^2) sum_e c_e sum_r q_re,
//   d loss / dx_rj = scale E / (K n^2) q_j (c_j - sum_e c_e q_e)      (times 1 - sigma_j).
// Balanced counts are all about K n / E and cancel in the gradient: they are taken less that
// number, which changes nothing as the shares sum to 1.
//
// Forward.  Workgroup i takes a span of rows; a row by a team of LANES lanes that hold R experts
// each, so that a lane sums the shares of its own experts over rows in registers (binary32, of at
// most 64 rows of a team), and counts go to LDS as integers, whose additions may come in any
// order.  At the end of each sequence's part of the span the sums of a wavefront's teams, up to
// eight, are joined in binary32 (three more roundings), then the wavefronts' in their order, in
// binary64.  A sequence within the span is finished there: by the workgroup, or one of few rows by
// a wavefront alone, so that several are worked on at once.  Of others the parts go to scratch, in
// binary32 beside their counts (a rounding of 2^-24 of each part, where 64 additions have made as
// many), and a second kernel joins them in the order of the spans, in binary64: the result is the
// same every time.
//
// Gradient: a row by a team as well, a lane keeps its experts' counts of the sequence that its row
// is in.
//
// What bounds them.  65536 x 256 bfloat16 sigmoid in 24 sequences takes 18 us, its 36 MB 5.2 at
// 6.9 TB/s: the arithmetic (an exponential and a reciprocal an element, about 14 instructions; 7 us
// of it), the chain ahead of and behind the rows (5 us, a batch of 16 rows) and the join, a launch
// (5 us).  The gradient of 65536 x 256 binary32 takes 26 us for 134 MB, a large copy's rate; of
// bfloat16 18 with softmax shares and 20 with sigmoids for 67 MB (a copy of as much 13.4): 890 and
// 1030 vector instructions a wavefront, 13 and 16 us of them on all SIMDs at 2.4 GHz.
#include <type_traits>

#include "experts.hpp"
#include "kernels.h"

namespace osm {

constexpr int BL_BLOCK = 256;   // of the gradient
constexpr int BL_WAVES = BL_BLOCK / 64;
constexpr int SPAN_WAVES = 16;  // of a span's workgroup
constexpr int BL_ADDED = 64;    // rows of a team whose shares are added in binary32

// A sequence's part of a span in scratch: for each expert the sum of its shares (binary32, upper
// word) and its count, then the rows that took part.  Slot 2 i is of the sequence that span i has
// from the span before, slot 2 i + 1 of the one that begins in it and goes on.
struct BalanceSpans {
    int64_t rows;      // of a span
    uint32_t spans;
    uint64_t* slots;   // spans * 2 * (E + 1)
    // of slot 2 i + 1: its sequence, or -1; the last span that has it; how many parts of its
    // experts are joined
    int4* leads;
    double* dots;      // 4 a span, 16 of the first: sums of counts times mean shares of those parts
};

__device__ __forceinline__ int64_t inside(const BalanceRows& a, int64_t v) {
    return v < 0 ? 0 : v > a.N ? a.N : v;
}
__device__ __forceinline__ int64_t seq_start(const BalanceRows& a, int64_t s) {
    if (!a.starts) return s == 0 ? 0 : a.N;
    return inside(a, a.starts[s]);
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
        const bool behind = s < hi && inside(a, a.starts[s + 1]) > row;
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

// Where sequences begin and end, by the whole wavefront: 64 of them in its lanes.
struct Sequences {
    int64_t base = 0;
    int32_t from = 0, to = 0;  // of sequence base + lane

    __device__ __forceinline__ void load(const BalanceRows& a, int64_t s) {
        base = s;
        if (!a.starts) {
            from = 0, to = (int32_t)a.N;
            return;
        }
        const int64_t i = s + (threadIdx.x & 63);
        const int32_t v = a.starts[i < a.S ? i : a.S], w = a.starts[i < a.S ? i + 1 : a.S];
        from = (int32_t)inside(a, v);
        to = (int32_t)inside(a, w);
        to = to > from ? to : from;
    }
    // The first one that ends behind `row`.
    __device__ __forceinline__ int64_t after(const BalanceRows& a, int64_t row) {
        if (a.S <= 64) {
            load(a, 0);
            const uint64_t who = __ballot((threadIdx.x & 63) < a.S && to > row);
            return who ? __builtin_ctzll(who) : a.S;
        }
        const int64_t s = seq_after(a, row);
        load(a, s);
        return s;
    }
    __device__ __forceinline__ void bounds(const BalanceRows& a, int64_t s, int64_t& begin,
                                           int64_t& end) {
        if (s - base >= 64) load(a, s);
        begin = __builtin_amdgcn_readlane(from, (int)(s - base));
        end = __builtin_amdgcn_readlane(to, (int)(s - base));
    }
};

// Shares of a row (see above) times a number: returns that times the factor.  For the gradient
// also 1 - sigma of each expert.
template <int LANES, int R, bool SLOPE>
__device__ __forceinline__ float shares(const float (&x)[R], bool sigmoid, float (&q)[R],
                                        float (&slope)[R]) {
    float sum = 0.0f;
    if (sigmoid) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const float e = exp2_hw(-x[j] * kLog2e);
            q[j] = __builtin_amdgcn_rcpf(1.0f + e);
            if constexpr (SLOPE) slope[j] = x[j] > 0.0f ? e * q[j] : 1.0f - q[j];
            sum += q[j];
        }
        sum = group_sum<LANES>(sum);
        if (__ballot(sum < 0x1p-60f) != 0) {  // only logits far below 0
            float m = x[0];
#pragma unroll
            for (int j = 1; j < R; ++j) m = fmaxf(m, x[j]);
            m = group_max<LANES>(m);
            const bool low = sum < 0x1p-60f;
            float t = 0.0f, p[R];
#pragma unroll
            for (int j = 0; j < R; ++j) {  // x < 0, where the sigmoid is e^x
                p[j] = exp2_hw((x[j] - m) * kLog2e);
                t += p[j];
            }
            t = group_sum<LANES>(t);
            sum = low ? t : sum;
#pragma unroll
            for (int j = 0; j < R; ++j) q[j] = low ? p[j] : q[j];
        }
    } else {
        float m = x[0];
#pragma unroll
        for (int j = 1; j < R; ++j) m = __builtin_elementwise_maximum(m, x[j]);
        // The rounding of m log2(e) is the same in all shares and small below 2^22.  From there on
        // it would not be, and the product itself may leave binary32: such a row's differences
        // are taken first (for all rows that is an operation more an element).
        m = team_maximum<LANES>(m);
        const float S = m * kLog2e;
        const bool far = !(__builtin_fabsf(S) < 0x1p22f);
        if (__builtin_expect(__ballot(far) != 0, 0)) {
            const float by = far ? m : 0.0f, S1 = far ? 0.0f : S;
#pragma unroll
            for (int j = 0; j < R; ++j) q[j] = exp2_hw(__builtin_fmaf(x[j] - by, kLog2e, -S1));
        } else {
#pragma unroll
            for (int j = 0; j < R; ++j) q[j] = exp2_hw(__builtin_fmaf(x[j], kLog2e, -S));
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if constexpr (SLOPE) slope[j] = 1.0f;
            sum += q[j];
        }
        sum = group_sum<LANES>(sum);
    }
    return __builtin_amdgcn_rcpf(sum);
}

// A team's rows as they come from memory, every so many-th of a span: their experts, and the lane's
// first index (every lane loads one).  Places are counted from the span's first row in 32 bits, and
// rows behind the last one are that.
template <typename T, int LANES, int R, int VEC>
struct TeamRows {
    RawExperts<T, LANES, R, VEC> raw;
    int32_t first;
    const char *x, *idx;           // of the span's first row
    uint32_t at, at_last, at_step;  // in bytes
    uint32_t i, i_last, i_step;

    __device__ __forceinline__ void span(const BalanceRows& a, int64_t r0) {
        x = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + r0 * a.E);
        idx = reinterpret_cast<const char*>(a.idx + r0 * a.K);
    }
    // From row r of the span on, in steps of `step`, to row end - 1.
    __device__ __forceinline__ void begin(const BalanceRows& a, uint32_t r, uint32_t step,
                                          uint32_t end, int lane) {
        const uint32_t xb = (uint32_t)a.E * (uint32_t)sizeof(T), ib = (uint32_t)a.K * 4;
        r = r < end ? r : end - 1;
        const uint32_t l = (uint32_t)(lane < a.K ? lane : 0) * 4;
        at = r * xb, at_last = (end - 1) * xb, at_step = step * xb;
        i = r * ib + l, i_last = (end - 1) * ib + l, i_step = step * ib;
        fetch(a, lane);
    }
    __device__ __forceinline__ void fetch(const BalanceRows& a, int lane) {
        raw.load(x, at, a.E, lane);
        first = *reinterpret_cast<const int32_t*>(idx + i);
        at = at + at_step < at_last ? at + at_step : at_last;
        i = i + i_step < i_last ? i + i_step : i_last;
    }
};

// Whether one of a row's indices is an expert, for a team that has them LANES at a time, the
// first ones in `first`.  COUNT: they are counted.
template <int LANES, bool COUNT>
__device__ __forceinline__ bool takes_part(const BalanceRows& a, int64_t row, bool live, int lane,
                                           int team, int32_t first, int32_t* counts) {
    bool in = live && lane < a.K && (uint32_t)first < (uint32_t)a.E;
    if (COUNT && in) atomicAdd(counts + first, 1);
    if (LANES < 64 && a.K > LANES) {
        for (int k = LANES; k < a.K; k += LANES) {  // uniform
            const int32_t e = live && k + lane < a.K ? a.idx[row * a.K + k + lane] : -1;
            const bool is = (uint32_t)e < (uint32_t)a.E;
            if (COUNT && is) atomicAdd(counts + e, 1);
            in = in || is;
        }
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

template <typename T, int LANES, int R, int VEC, bool FULL>
__global__ __launch_bounds__(64 * SPAN_WAVES) void balance_spans(
    const BalanceRows a, const BalanceSpans b) {
    constexpr int ROWS = 64 / LANES, WAVES = SPAN_WAVES, TEAMS = WAVES * ROWS;
    constexpr int THREADS = 64 * WAVES;
    __shared__ float acc[WAVES][LANES * R];  // a wavefront's sums; its counts, where it is alone
    __shared__ double sums[LANES * R];
    __shared__ int32_t counts[LANES * R];
    __shared__ int32_t part_rows[WAVES];
    __shared__ double part[WAVES];
    const int tid = threadIdx.x, lane = tid % LANES, team = (tid & 63) / LANES;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int E = a.E;
    const int64_t r0 = blockIdx.x * b.rows, r1 = r0 + b.rows < a.N ? r0 + b.rows : a.N;
    // a row is on its way while the one before is worked on, the first one before its sequence
    // is known
    TeamRows<T, LANES, R, VEC> rows;
    rows.span(a, r0);
    if (r0 < r1) rows.begin(a, wv * ROWS + team, TEAMS, (uint32_t)(r1 - r0), lane);
    // its sequences: those that end behind r0 (all that end at row 0 are the first span's)
    Sequences seq;
    int64_t begin = 0;
    if (blockIdx.x == 0) seq.load(a, 0);
    else begin = seq.after(a, r0);
    int4 lead = {-1, 0, 0, 0};
    bool ahead = true;  // `rows` has the span's first ones
    // 64 sequences at a time: first those that the workgroup takes together, then the ones of few
    // rows, within the span and not all of it, that a wavefront takes alone
    for (bool more = true; more; seq.load(a, seq.base + 64)) {
        uint64_t todo, few;
        {
            const int64_t s = seq.base + (tid & 63), n = seq.to - seq.from;
            const bool ok = s >= begin && s < a.S &&
                            (seq.from < r1 || (seq.from == r1 && n == 0));
            const bool in = ok && n < r1 - r0 && seq.from >= r0 && seq.to <= r1;
            few = __ballot(in && n <= 8 * ROWS);
            // (up to 32 rows of a team where there are several: a workgroup has a fixed 3.5 us
            // for each, a wavefront 10 at most; 65536 x 64 in 1000 sequences 30.3 us, so 17.8)
            const uint64_t mid = __ballot(in && n <= 32 * ROWS);
            if (__builtin_popcountll(mid & ~few) >= 3) few = mid;
            todo = __ballot(ok) & ~few;
            more = __ballot(ok) >> 63;
        }
        for (int phase = 0; phase < 2; ++phase) {
            const bool alone = phase == 1;
            // (every so many-th of them is this wavefront's)
            if (alone) todo = few & 0x0001000100010001ull << wv;
            for (; todo != 0; todo &= todo - 1) {
                const int at = __builtin_ctzll(todo);
                const int64_t s = seq.base + at;
                const int64_t from = __builtin_amdgcn_readlane(seq.from, at);
                const int64_t to = __builtin_amdgcn_readlane(seq.to, at);
                const bool before = from < r0, behind = to > r1;
                const int64_t p0 = from > r0 ? from : r0, p1 = to < r1 ? to : r1;
                int32_t* const own = alone ? reinterpret_cast<int32_t*>(acc[wv]) : counts;
                const int64_t step = alone ? ROWS : TEAMS;
                int64_t row0 = p0 + (alone ? 0 : wv * ROWS);
                if ((!ahead || p0 != r0 || p1 != r1 || alone) && p0 < p1)
                    rows.begin(a, (uint32_t)(row0 + team - r0), (uint32_t)step,
                               (uint32_t)(p1 - r0), lane);
                ahead = false;
                if (alone) {
                    for (int e = tid & 63; e < LANES * R; e += 64) own[e] = 0;
                    wave_sync();
                } else {
                    for (int e = tid; e < LANES * R; e += THREADS) own[e] = 0;
                    __syncthreads();
                }
                float sum[R];
                int32_t n = 0;
#pragma unroll
                for (int j = 0; j < R; ++j) sum[j] = 0.0f;
                for (; row0 < p1; row0 += step) {
                    const int64_t row = row0 + team;
                    const RawExperts<T, LANES, R, VEC> raw = rows.raw;
                    const int32_t first = rows.first;
                    rows.fetch(a, lane);
                    float x[R], q[R], none[R];
                    raw.template widen<FULL>(x, E, lane);
                    const bool in =
                        takes_part<LANES, true>(a, row, row < p1, lane, team, first, own);
                    float r = shares<LANES, R, false>(x, a.sigmoid, q, none);
                    if (__ballot(!in) != 0) {  // (its shares may be anything)
                        r = in ? r : 0.0f;
#pragma unroll
                        for (int j = 0; j < R; ++j) q[j] = in ? q[j] : 0.0f;
                    }
#pragma unroll
                    for (int j = 0; j < R; ++j) sum[j] = __builtin_fmaf(q[j], r, sum[j]);
                    n += in && lane == 0;
                }
                n = (int32_t)group_sum<64>((float)n);
#pragma unroll
                for (int j = 0; j < R; ++j) sum[j] = sum_of_teams<LANES>(sum[j]);
                if (alone) {
                    wave_sync();
                    const double rn = n > 0 ? 1.0 / (double)n : 0.0;
                    double dot = 0.0;
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        const int e = expert<LANES, VEC>(lane, j);
                        if (team != 0 || e >= E) continue;
                        const double mean = (double)sum[j] * rn;
                        const int32_t c = own[e];
                        a.probs[s * E + e] = (float)mean;
                        a.counts[s * E + e] = c;
                        dot += (double)c * mean;
                    }
                    dot = group_sum<64>(dot);
                    if ((tid & 63) == 0) {
                        a.loss[s] = (float)((double)a.scale * E / a.K * rn * dot);
                        a.rows[s] = n;
                    }
                    wave_sync();
                    continue;
                }
                // the teams' sums, wavefront by wavefront
#pragma unroll
                for (int j = 0; j < R; ++j)
                    if (team == 0) acc[wv][expert<LANES, VEC>(lane, j)] = sum[j];
                if ((tid & 63) == 0) part_rows[wv] = n;
                __syncthreads();
                n = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) n += part_rows[w];
                uint64_t* const slot =
                    b.slots + ((int64_t)blockIdx.x * 2 + (before ? 0 : 1)) * (E + 1);
                for (int e = tid; e < E; e += THREADS) {
                    double v = 0.0;
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) v += (double)acc[w][e];
                    if (before || behind)
                        slot[e] = (uint64_t)__float_as_uint((float)v) << 32 | (uint32_t)counts[e];
                    else
                        sums[e] = v;
                }
                if (before || behind) {
                    if (tid == 0) slot[E] = (uint32_t)n;
                    if (!before) lead = int4{(int32_t)s, (int32_t)((to - 1) / b.rows), 0, 0};
                } else {
                    __syncthreads();
                    finish<THREADS>(a, s, sums, counts, n, part);
                }
                __syncthreads();
            }
        }
        if (more) __syncthreads();
    }
    if (tid == 0 && b.spans > 1) b.leads[blockIdx.x] = lead;
}

// Sequences that more than one span has: workgroup (i, part) joins 64 COLS experts of the one that
// begins in span i.  Each wavefront takes every so many-th slot, COLS experts a lane, eight slots
// in flight.  The last part of a sequence to arrive has its loss.  All rows as one sequence are
// joined 64 experts a workgroup (65536 x 256: 17.8 us, with one workgroup 22.0); of others a
// workgroup takes 256, so that few are launched in vain (in 24 sequences 17.8 us, with four
// workgroups a span 22.4).
constexpr int JOIN_COLS = 4;  // at most

template <int COLS>
__global__ __launch_bounds__(1024) void balance_join(const BalanceRows a, const BalanceSpans b) {
    constexpr int WAVES = 16, DEEP = 8, WIDE = 64 * COLS;
    __shared__ double stripe[WAVES][WIDE];
    __shared__ int32_t stripe_counts[WAVES][WIDE];
    __shared__ int32_t rows[WAVES];
    __shared__ double dots[WAVES];
    const int4 lead = b.leads[blockIdx.x];
    if (lead.x < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, E = a.E;
    const int e0 = (int)blockIdx.y * WIDE;
    // slots: the second one of this span, the first ones of the following
    const int64_t i0 = blockIdx.x;
    const int last = (lead.y < (int)b.spans ? lead.y : (int)b.spans - 1) - (int)i0;
    auto slot = [&](int j) { return b.slots + (j == 0 ? i0 * 2 + 1 : (i0 + j) * 2) * (E + 1); };
    double v[COLS];
    int32_t c[COLS], n = 0;
#pragma unroll
    for (int k = 0; k < COLS; ++k) v[k] = 0.0, c[k] = 0;
    for (int j = tid; j <= last; j += 64 * WAVES) n += (int32_t)(uint32_t)slot(j)[E];
    for (int j0 = wv; j0 <= last; j0 += WAVES * DEEP) {
        uint64_t w[DEEP][COLS];
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int j = j0 + d * WAVES;
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                const int e = e0 + lane + 64 * k;
                w[d][k] = j <= last && e < E ? slot(j)[e] : 0;
            }
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                v[k] += (double)__uint_as_float((uint32_t)(w[d][k] >> 32));
                c[k] += (int32_t)(uint32_t)w[d][k];
            }
        }
    }
    for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
    if (lane == 0) rows[wv] = n;
#pragma unroll
    for (int k = 0; k < COLS; ++k) {
        stripe[wv][lane + 64 * k] = v[k];
        stripe_counts[wv][lane + 64 * k] = c[k];
    }
    __syncthreads();
    n = 0;
    for (int w = 0; w < WAVES; ++w) n += rows[w];
    const int64_t s = lead.x;
    const double rn = n > 0 ? 1.0 / (double)n : 0.0;
    double dot = 0.0;
    if (tid < WIDE && e0 + tid < E) {
        double t = 0.0;
        int32_t m = 0;
        for (int w = 0; w < WAVES; ++w) {
            t += stripe[w][tid];
            m += stripe_counts[w][tid];
        }
        t *= rn;
        a.probs[s * E + e0 + tid] = (float)t;
        a.counts[s * E + e0 + tid] = m;
        dot = (double)m * t;
    }
    dot = group_sum<64>(dot);
    if (lane == 0) dots[wv] = dot;
    __syncthreads();
    if (tid != 0) return;
    dot = 0.0;
    for (int w = 0; w < COLS; ++w) dot += dots[w];
    const int parts = gridDim.y;
    if (parts > 1) {
        uint64_t* const at = reinterpret_cast<uint64_t*>(b.dots + i0 * 4);
        __hip_atomic_store(at + blockIdx.y, __builtin_bit_cast(uint64_t, dot), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const int32_t arrived = __hip_atomic_fetch_add(&b.leads[i0].z, 1, __ATOMIC_RELAXED,
                                                       __HIP_MEMORY_SCOPE_AGENT);
        if (arrived != parts - 1) return;
        dot = 0.0;
        for (int i = 0; i < parts; ++i)
            dot += __builtin_bit_cast(double, __hip_atomic_load(at + i, __ATOMIC_RELAXED,
                                                                __HIP_MEMORY_SCOPE_AGENT));
    }
    a.loss[s] = (float)((double)a.scale * E / a.K * rn * dot);
    a.rows[s] = n;
}

template <typename T, int LANES, int R, int VEC, bool FULL>
__global__ __launch_bounds__(BL_BLOCK) void balance_grad(const BalanceRows a, int64_t span) {
    constexpr int ROWS = 64 / LANES, TEAMS = BL_WAVES * ROWS;
    const int tid = threadIdx.x, lane = tid % LANES, wv = tid >> 6, team = (tid & 63) / LANES;
    const int E = a.E;
    const int64_t r0 = blockIdx.x * span, r1 = r0 + span < a.N ? r0 + span : a.N;
    // a row is on its way while the one before is worked on, the first one while its sequence
    // is looked for
    TeamRows<T, LANES, R, VEC> rows;
    rows.span(a, r0);
    rows.begin(a, wv * ROWS + team, TEAMS, (uint32_t)(r1 - r0), lane);
    int64_t row = r0 + wv * ROWS + team;
    // the sequence of this lane's row: none from s_end on
    int64_t s = 0, s_from = INT64_MAX, s_end = INT64_MAX;
    float c[R], f = 0.0f;
    auto enter = [&] {
        const double n = (double)a.rows[s], mean = (double)a.K * n / E;
        const double g = (double)a.dloss[s] * a.scale * E;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int e = expert<LANES, VEC>(lane, j);
            const int32_t v = a.counts[s * E + (FULL || e < E ? e : 0)];
            c[j] = FULL || e < E ? (float)((double)v - mean) : 0.0f;
        }
        f = n > 0.0 ? (float)(g / (a.K * n * n)) : 0.0f;
    };
#pragma unroll
    for (int j = 0; j < R; ++j) c[j] = 0.0f;
    {
        Sequences seq;
        s = seq.after(a, r0 + wv * ROWS);
        if (s < a.S) {
            seq.bounds(a, s, s_from, s_end);
            enter();
        }
    }
    for (int64_t row0 = r0 + wv * ROWS; row0 < r1; row0 += TEAMS) {
        const RawExperts<T, LANES, R, VEC> raw = rows.raw;
        const int32_t first = rows.first;
        rows.fetch(a, lane);
        const bool live = row < r1;
        float x[R], q[R], slope[R];
        raw.template widen<FULL>(x, E, lane);
        const bool in = takes_part<LANES, false>(a, row, live, lane, team, first, nullptr);
        if (live && row >= s_end) {  // another sequence
            while (s < a.S && (s_end = seq_start(a, s + 1)) <= row) ++s;
            if (s < a.S) {
                s_from = seq_start(a, s);
                enter();
            } else {
                s_from = s_end = INT64_MAX;
            }
        }
        const bool part = in && row >= s_from;
        const float r = shares<LANES, R, true>(x, a.sigmoid, q, slope);
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < R; ++j) dot = __builtin_fmaf(c[j], q[j], dot);
        dot = group_sum<LANES>(dot) * r;
        float d[R];
        const float k = r * f;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            d[j] = q[j] * k * (c[j] - dot);
            if (a.sigmoid) d[j] *= slope[j];
        }
        if (__ballot(!part) != 0) {
#pragma unroll
            for (int j = 0; j < R; ++j) d[j] = part ? d[j] : 0.0f;
        }
        if (live) store_experts<T, LANES, R, VEC>(static_cast<T*>(a.dx) + row * E, E, lane, d);
        row += TEAMS;
    }
}

// Lanes of a row: 8 experts a lane, in at least 8 and at most 64 lanes (16 experts a lane are not
// faster at any size tried).
static int balance_lanes(int E) {
    int lanes = 8;
    while (lanes < 64 && lanes * 8 < E) lanes *= 2;
    return lanes;
}

// Rows of a span: one for all where a team has at most four, else a workgroup a CU, or for every
// second one where a team would have less than four (one workgroup joins a sequence, and for longer
// the more spans it has: 16384 x 256 in 128 of them 14.9 us, in 256 17.6), and at most BL_ADDED a
// team.
static int64_t balance_span(int64_t N, int E, int cus) {
    const int64_t teams = SPAN_WAVES * (64 / balance_lanes(E));
    if (N <= 4 * teams) return 4 * teams;
    auto of = [&](int64_t spans) { return ((N + spans - 1) / spans + teams - 1) / teams * teams; };
    int64_t rows = of(cus);
    if (rows < 4 * teams) rows = of(cus / 2 + 1) < 4 * teams ? of(cus / 2 + 1) : 4 * teams;
    return rows < BL_ADDED * teams ? rows : BL_ADDED * teams;
}

static uint32_t balance_spans_of(int64_t N, int64_t rows) {
    return N > 0 ? (uint32_t)((N + rows - 1) / rows) : 1;
}

static size_t slots_bytes(size_t spans, size_t E) {
    return (spans * 2 * (E + 1) * 8 + 255) / 256 * 256;
}

size_t balance_scratch_bytes(int64_t N, int64_t E, int cus) {
    const size_t spans = balance_spans_of(N, balance_span(N, (int)E, cus));
    return spans > 1 ? slots_bytes(spans, (size_t)E) + spans * (sizeof(int4) + 4 * sizeof(double)) +
                           12 * sizeof(double)
                     : 0;
}

// Teams of LANES lanes with R experts each, VEC neighbours at a time: f is called with them as
// constants.
template <bool VEC4, typename F>
static void with_team(int E, F f) {
    constexpr int VEC = VEC4 ? 4 : 1;
    auto r = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        auto call = [&](auto n) { f(lanes, n, std::integral_constant<int, VEC>{}); };
        if constexpr (L == 8) {
            if constexpr (VEC == 1) {
                if (E <= 8) return call(std::integral_constant<int, 1>{});
                if (E <= 16) return call(std::integral_constant<int, 2>{});
            }
            if (E <= 32) return call(std::integral_constant<int, 4>{});
        }
        if constexpr (L == 64)
            if (E > 512) return call(std::integral_constant<int, 16>{});
        call(std::integral_constant<int, 8>{});
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
    b.slots = static_cast<uint64_t*>(scratch);
    b.leads = reinterpret_cast<int4*>(static_cast<char*>(scratch) +
                                      slots_bytes(b.spans, (size_t)a.E));
    b.dots = reinterpret_cast<double*>(b.leads + b.spans);
    auto go = [&](auto lanes, auto r, auto vec) {
        constexpr int R = decltype(r)::value;
        constexpr int L = decltype(lanes)::value, V = decltype(vec)::value;
        const dim3 grid(b.spans), block(64 * SPAN_WAVES);
        if (a.E == L * R)
            hipLaunchKernelGGL((balance_spans<T, L, R, V, true>), grid, block, 0, st, a, b);
        else
            hipLaunchKernelGGL((balance_spans<T, L, R, V, false>), grid, block, 0, st, a, b);
    };
    if (four(a, sizeof(T), false)) with_team<true>(a.E, go);
    else with_team<false>(a.E, go);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || b.spans == 1) return e;
    const int cols = (a.E + 63) / 64;
#define OSM_JOIN(C)                                                                         \
    hipLaunchKernelGGL((balance_join<C>), dim3(a.starts ? b.spans : 1, (cols + C - 1) / C), \
                       dim3(1024), 0, st, a, b)
    if (cols <= 1 || !a.starts) OSM_JOIN(1);
    else if (cols <= 2) OSM_JOIN(2);
    else OSM_JOIN(JOIN_COLS);
#undef OSM_JOIN
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_balance_bwd_t(const BalanceRows& a, hipStream_t st) {
    const int64_t teams = BL_BLOCK / balance_lanes(a.E);
    const int64_t want = (a.N + teams - 1) / teams, most = 8 * (int64_t)a.cus;
    const int64_t blocks = want < most ? want : most;
    int64_t span = (a.N + blocks - 1) / blocks;
    if (span > 1 << 16) span = 1 << 16;  // (places within it in 32 bits)
    auto go = [&](auto lanes, auto r, auto vec) {
        constexpr int L = decltype(lanes)::value, R = decltype(r)::value, V = decltype(vec)::value;
        const dim3 grid((unsigned)((a.N + span - 1) / span)), block(BL_BLOCK);
        if (a.E == L * R)
            hipLaunchKernelGGL((balance_grad<T, L, R, V, true>), grid, block, 0, st, a, span);
        else
            hipLaunchKernelGGL((balance_grad<T, L, R, V, false>), grid, block, 0, st, a, span);
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
