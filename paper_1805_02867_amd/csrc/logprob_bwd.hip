// The gradient of log probabilities and entropy with respect to the logits, and the plan of
// the forward kernels.
//
// With p_j = 2^{(x_j - m) c} / (1 + s) from the row's (m, s), G the sum of the tokens' gradients
// and h the entropy's:
//   dx_j = (-p_j G - h p_j (ln p_j + H) + sum of g over the tokens that are j) / temperature
//        = p_j (alpha + beta (x_j - m) c) + ...,  alpha, beta a row's constants.
// Every element gets the first part; the lane that stored a token's element then stores it
// again, from binary64: where p_t is close to 1, g (1 - p_t) is formed with
// 1 - p_t = -expm1(ln p_t), which the difference of binary32 numbers has lost.
//
// What bounds it is memory: an element is read and written once, with a subtraction, an
// exponential and four other operations.
#include "kernels.h"
#include "wide.hpp"

namespace osm {

constexpr int LB_BLOCK = 256;
constexpr int LB_U = 4;  // vectors a lane

// Sixteen bytes at any element's address.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <typename T>
__device__ __forceinline__ Vec<T> load_any(const T* p) {
    const u32x4 q = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
    if constexpr (sizeof(T) == 2)
        return Vec<T>::unpack(q);
    else
        return Vec<T>{{__uint_as_float(q.x), __uint_as_float(q.y), __uint_as_float(q.z),
                       __uint_as_float(q.w)}};
}

// A row's constants.
struct GradRow {
    float m, c, alpha, beta;
    bool zero;  // no gradient comes in
};

template <bool ENT>
__device__ __forceinline__ float grad_of(const GradRow& r, float x) {
    const float t = (x - r.m) * r.c;
    const float p = exp2_hw(t);
    // (-inf has no weight: -200 stands for what is as small, so that 0 times it is 0)
    return ENT ? p * __builtin_fmaf(r.beta, __builtin_fmaxf(t, -200.0f), r.alpha) : p * r.alpha;
}

// Piece b of a row by TR lanes: U vectors a lane from the first 16-byte boundary of dx on,
// piece 0 with the elements in front of it and behind the last whole vector.
template <typename T, int TR, bool ENT>
__global__ __launch_bounds__(LB_BLOCK) void logprob_grad(const LogprobGrad a, uint32_t pieces) {
    constexpr int E = Vec<T>::N, U = LB_U, TEAMS = LB_BLOCK / TR;
    const int lane = threadIdx.x & 63;
    const int tr = threadIdx.x % TR;
    const int64_t unit = (int64_t)blockIdx.x * TEAMS +
                         (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TR) : 0);
    const int64_t row = unit / pieces;
    if (row >= a.N) return;  // whole wavefronts; no barrier follows
    const uint32_t piece = (uint32_t)(unit - row * pieces);
    const T* xr = static_cast<const T*>(a.x) + row * a.ldx;
    T* dr = static_cast<T*>(a.dx) + row * a.lddx;
    int64_t head = (int64_t)(((16 - (((uintptr_t)dr) & 15)) & 15) / sizeof(T));
    head = head < a.V ? head : a.V;
    const int64_t nvec = (a.V - head) / E;
    const int64_t v0 = (int64_t)piece * (TR * U);
    const int extras = piece == 0 ? (int)(a.V - nvec * E) : 0;  // head and tail, below 2 E
    // place of the i-th of them
    auto extra = [&](int i) { return i < head ? (int64_t)i : nvec * E + i; };

    // the elements first; lanes past the row load its last vector and do not store it
    Vec<T> buf[U];
    if (v0 < nvec) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t v = v0 + tr + i * TR;
            buf[i] = load_any<T>(xr + head + (v < nvec ? v : nvec - 1) * E);
        }
    }
    const float ex = tr < extras ? load1(xr + extra(tr)) : 0.0f;

    int32_t tok = -1;
    float g = 0.0f;
    if (lane < a.T) {
        tok = a.tokens[row * a.T + lane];
        const bool in = tok >= 0 && (int64_t)tok < a.V;
        tok = in ? tok : -1;
        if (in) g = a.dlogp[row * a.T + lane];
    }
    const double G = group_sum<64>((double)g);
    const float h = ENT ? a.dentropy[row] : 0.0f;
    const float m = a.stats[row * 2], s = a.stats[row * 2 + 1];
    const double ln_d = log1p((double)s), rd = 1.0 / (1.0 + (double)s);
    const double H = ENT ? (double)a.entropy[row] : 0.0;
    GradRow r;
    r.m = m;
    r.c = a.c;
    r.zero = __builtin_amdgcn_ballot_w64(!(g == 0.0f)) == 0 && h == 0.0f;
    r.alpha = (float)(-a.inverse * rd * (G + (ENT ? (double)h * (H - ln_d) : 0.0)));
    r.beta = ENT ? (float)(-a.inverse * rd * (double)h * 0.69314718055994530942) : 0.0f;

#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t v = v0 + tr + i * TR;
        if (v >= nvec) continue;
        Vec<T> out;
#pragma unroll
        for (int e = 0; e < E; ++e) out.v[e] = r.zero ? 0.0f : grad_of<ENT>(r, buf[i].v[e]);
        out.store_nt(dr + head + v * E);
    }
    if (tr < extras) store1(dr + extra(tr), r.zero ? 0.0f : grad_of<ENT>(r, ex));
    if (r.zero) return;

    // the tokens' own elements
    for (int i = 0; i < a.T; ++i) {
        const int32_t t = __builtin_amdgcn_readlane(tok, i);
        if (t < 0) continue;
        // who stored it
        int64_t at;
        const int64_t v = (int64_t)t >= head ? (t - head) / E : -1;
        if (v < 0 || v >= nvec) {
            if (piece != 0) continue;
            at = v < 0 ? t : t - nvec * E;
        } else {
            if (v < v0 || v >= v0 + TR * U) continue;
            at = (v - v0) % TR;
        }
        const uint64_t same = __builtin_amdgcn_ballot_w64(tok == t);
        if ((same & ((1ull << i) - 1)) != 0) continue;  // done with its first place
        const double gt = group_sum<64>(tok == t ? (double)g : 0.0);
        const double lp = ((double)load1(xr + t) - (double)m) * a.inverse - ln_d;
        const double p = exp(lp);
        double d = gt * -expm1(lp) - p * (G - gt);
        if (ENT && p > 0.0) d -= (double)h * p * (lp + H);
        if (tr == (int)at) store1(dr + t, (float)(d * a.inverse));
    }
}

template <typename T>
hipError_t launch_logprob_bwd_t(const LogprobGrad& a, hipStream_t st) {
    constexpr int E = Vec<T>::N;
    const int64_t nv = a.V / E;  // at least the whole vectors
    const bool wave = nv <= 64 * LB_U;
    const int64_t tr = wave ? 64 : LB_BLOCK;
    int64_t pieces = (nv + tr * LB_U - 1) / (tr * LB_U);
    if (pieces < 1) pieces = 1;
    const int64_t teams = LB_BLOCK / tr;
    // a launch has fewer than 2^32 threads: rows beyond that in another one
    const int64_t most = ((int64_t)1 << 23) / pieces > 0 ? ((int64_t)1 << 23) / pieces : 1;
    LogprobGrad b = a;
    for (int64_t row0 = 0; row0 < a.N; row0 += most) {
        b.N = a.N - row0 < most ? a.N - row0 : most;
        b.x = static_cast<const T*>(a.x) + row0 * a.ldx;
        b.dx = static_cast<T*>(a.dx) + row0 * a.lddx;
        b.tokens = a.tokens ? a.tokens + row0 * a.T : nullptr;
        b.dlogp = a.dlogp ? a.dlogp + row0 * a.T : nullptr;
        b.stats = a.stats + row0 * 2;
        b.entropy = a.entropy ? a.entropy + row0 : nullptr;
        b.dentropy = a.dentropy ? a.dentropy + row0 : nullptr;
        const dim3 grid((unsigned)((b.N * pieces + teams - 1) / teams)), block(LB_BLOCK);
        const uint32_t n = (uint32_t)pieces;
        if (wave && a.dentropy)
            hipLaunchKernelGGL((logprob_grad<T, 64, true>), grid, block, 0, st, b, n);
        else if (wave)
            hipLaunchKernelGGL((logprob_grad<T, 64, false>), grid, block, 0, st, b, n);
        else if (a.dentropy)
            hipLaunchKernelGGL((logprob_grad<T, LB_BLOCK, true>), grid, block, 0, st, b, n);
        else
            hipLaunchKernelGGL((logprob_grad<T, LB_BLOCK, false>), grid, block, 0, st, b, n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_logprob_bwd(const LogprobGrad& a, int dtype, hipStream_t st) {
    return dtype == 1 ? launch_logprob_bwd_t<bf16_t>(a, st) : launch_logprob_bwd_t<float>(a, st);
}

// Rows that a wavefront holds take one where there are enough of them to fill the chip; longer
// ones a workgroup of four or eight; rows that eight wavefronts do not hold, or too few to
// fill the chip, are split.
LogprobPlan logprob_plan(int64_t N, int64_t V, int K, int dtype, int cus) {
    const int64_t E = dtype == 1 ? 8 : 4;
    const int64_t nv = (V + E - 1) / E;
    const int64_t hold4 = 256 * 16, hold8 = 512 * 16;  // vectors
    LogprobPlan p{4, 1, V, N};
    int64_t S = (nv + hold8 - 1) / hold8;
    if (nv > 1024 && N < 2 * (int64_t)cus) {
        const int64_t want = (2 * (int64_t)cus + N - 1) / N, most = (nv + 511) / 512;
        const int64_t more = want < most ? want : most;
        S = S > more ? S : more;
    }
    if (S <= 1) {
        if (nv <= 1024 && (nv <= 64 || N >= 4 * (int64_t)cus)) p.W = 1;
        else p.W = nv <= hold4 ? 4 : 8;
        return p;
    }
    const int64_t vecs = (nv + S - 1) / S;
    p.chunk = vecs * E;
    p.S = (int)((V + p.chunk - 1) / p.chunk);
    p.W = vecs <= hold4 ? 4 : 8;
    // 2^16 chunks a launch, or one row
    const int64_t rows = ((int64_t)1 << 16) / p.S;
    p.rows = rows < 1 ? 1 : rows < N ? rows : N;
    (void)K;
    return p;
}

}  // namespace osm
