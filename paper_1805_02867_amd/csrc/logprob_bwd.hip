// The gradient of log probabilities and entropy with respect to the logits, and the plan of
// the forward kernels.
//
// With p_j = 2^{(x_j - m) c} / (1 + s) from the row's (m, s), G the sum of the tokens' gradients
// and h the entropy's:
//   dx_j = (-p_j G - h p_j (ln p_j + H) + sum of g over the tokens that are j) / temperature
//        = p_j (alpha + beta (x_j - m) c) + ...,  alpha, beta a row's constants.
// Every element gets the first part; then the tokens' elements are stored again, from binary64:
// where p_t is close to 1, g (1 - p_t) is formed with 1 - p_t = -expm1(ln p_t), which the
// difference of binary32 numbers has lost.
//
// What bounds it is memory: an element is read and written once, with a subtraction, an
// exponential and four other operations.  2048 x 128256 bfloat16 takes 180 us for 1.05 GB, 5.8 TB/s
// (a copy of as much 197), 1003 x 50257 binary32 with the entropy 70 us for 403 MB.  Of short
// rows it is the arithmetic that is not their elements' (G, 1 / (1 + s), alpha, the token's element),
// done by all lanes of a row's team: 100000 x 64 binary32 18 us (219 vector instructions for four
// rows, 9 us of them), 300000 x 20 bfloat16 43 (324, 39 us), 16385 x 1000 bfloat16 17 (341 a row,
// 9 us), binary32 27; copies of as much 9.9, 5.4, 12.3 and 24.6.
#include "kernels.h"
#include "wide.hpp"

namespace osm {

constexpr int LB_BLOCK = 256;
constexpr int LB_U = 4;     // vectors a lane
// Lanes of a row of up to 64 vectors: four rows a wavefront (100000 x 64 binary32 70.7 us with a
// wavefront a row, 19.1 so).
constexpr int LB_FEW = 16;

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
};

template <bool ENT>
__device__ __forceinline__ float grad_of(const GradRow& r, float x) {
    const float t = (x - r.m) * r.c;
    const float p = exp2_hw(t);
    // (-inf has no weight: -200 stands for what is as small, so that 0 times it is 0)
    return ENT ? p * __builtin_fmaf(r.beta, __builtin_fmaxf(t, -200.0f), r.alpha) : p * r.alpha;
}

// Piece b of a row by TR lanes: U vectors a lane from the first 16-byte boundary of dx on,
// piece 0 with the elements in front of it and behind the last whole vector.  (T <= TR.)
template <typename T, int TR, bool ENT>
__global__ __launch_bounds__(LB_BLOCK) void logprob_grad(const LogprobGrad a, uint32_t pieces) {
    constexpr int E = Vec<T>::N, U = LB_U, TEAMS = LB_BLOCK / TR;
    constexpr int TL = TR < 64 ? TR : 64;  // lanes of a row or piece in one wavefront
    const int lane = threadIdx.x % TL;
    const int tr = threadIdx.x % TR;
    const uint64_t team = TL == 64 ? ~0ull
                                   : ((1ull << TL) - 1) << ((threadIdx.x & 63) / TL * TL);
    int64_t row = blockIdx.x;
    uint32_t piece = 0;
    bool live = true;
    if constexpr (TR < 64) {  // (a row is one piece)
        row = row * TEAMS + threadIdx.x / TR;
        live = row < a.N;  // the others do the last row again, and store nothing
        row = live ? row : a.N - 1;
    } else {
        const int64_t unit =
            row * TEAMS + (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TR) : 0);
        row = unit / pieces;
        if (row >= a.N) return;  // whole wavefronts; no barrier follows
        piece = (uint32_t)(unit - row * pieces);
    }
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
    const float m = a.stats[row * 2], s = a.stats[row * 2 + 1];
    const float h = ENT ? a.dentropy[row] : 0.0f;
    const double H = ENT ? (double)a.entropy[row] : 0.0;
    // lane l has the l-th token
    int32_t tok = -1;
    float g = 0.0f;
    if (a.T > 0) {
        const int64_t at = row * a.T + (lane < a.T ? lane : 0);
        const int32_t t = a.tokens[at];
        const float v = a.dlogp[at];
        const bool in = lane < a.T && t >= 0 && (int64_t)t < a.V;
        tok = in ? t : -1;
        g = in ? v : 0.0f;
    }
    // those among this piece's elements
    const int64_t tv = (int64_t)tok >= head ? (tok - head) / E : nvec;  // (nvec: none)
    const bool here = tok >= 0 && (tv < nvec ? tv >= v0 && tv < v0 + TR * U : piece == 0);
    const bool any = __builtin_amdgcn_ballot_w64(here) != 0;
    const float tx = here ? load1(xr + tok) : 0.0f;

    const double G = group_sum<TL>((double)g), d1 = 1.0 + (double)s;
    const double rd0 = (double)__builtin_amdgcn_rcpf((float)d1), rd = rd0 * (2.0 - d1 * rd0);
    const double ln_d = ENT || any ? ln_1p(s) : 0.0;
    const bool zero = (__builtin_amdgcn_ballot_w64(!(g == 0.0f)) & team) == 0 && h == 0.0f;
    GradRow r;
    r.m = m;
    r.c = a.c;
    r.alpha = (float)(-a.inverse * rd * (G + (ENT ? (double)h * (H - ln_d) : 0.0)));
    r.beta = ENT ? (float)(-a.inverse * rd * (double)h * 0.69314718055994530942) : 0.0f;

#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t v = v0 + tr + i * TR;
        if (v >= nvec || !live) continue;
        Vec<T> out;
#pragma unroll
        for (int e = 0; e < E; ++e) out.v[e] = zero ? 0.0f : grad_of<ENT>(r, buf[i].v[e]);
        out.store_nt(dr + head + v * E);
    }
    if (tr < extras && live) store1(dr + extra(tr), zero ? 0.0f : grad_of<ENT>(r, ex));
    if (!any || (TR >= 64 && zero)) return;  // (the same in the piece's wavefronts)

    // The tokens' own elements, a lane each, by the piece's first wavefront once they are
    // stored.  A token that occurs twice is its first lane's.
    if constexpr (TR > 64) {
        __syncthreads();
        if (threadIdx.x >= 64) return;
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    double gt = 0.0;
    bool first = here;
    for (int i = 0; i < a.T; ++i) {
        const bool same = (TR < 64 ? __shfl(tok, i, TL) : __builtin_amdgcn_readlane(tok, i)) == tok;
        const float v = TR < 64 ? __shfl(g, i, TL) : lane_value(g, i);
        gt += same ? (double)v : 0.0;
        first = first && !(same && i < lane);
    }
    if (!first || zero || !live) return;
    // p and 1 - p: next to 1 by the series of e^lp - 1 (the first term left out 2^-26 of it), else
    // p as precise as the other elements' (the library's binary64 functions, with its logarithm
    // above: 2000 x 32000 bfloat16, 64 tokens a row, 56 us for 53)
    const double lp = ((double)tx - (double)m) * a.inverse - ln_d;
    double p = (double)exp2_hw((float)(lp * 1.4426950408889634074)), q = 1.0 - p;
    if (lp > -0.5) {
        q = 1.0 / 40320;
        q = __builtin_fma(q, lp, 1.0 / 5040);
        q = __builtin_fma(q, lp, 1.0 / 720);
        q = __builtin_fma(q, lp, 1.0 / 120);
        q = __builtin_fma(q, lp, 1.0 / 24);
        q = __builtin_fma(q, lp, 1.0 / 6);
        q = __builtin_fma(q, lp, 0.5);
        q = -lp * __builtin_fma(q, lp, 1.0);
        p = 1.0 - q;
    }
    double d = gt * q - p * (G - gt);
    if (ENT && p > 0.0) d -= (double)h * p * (lp + H);
    store1(dr + tok, (float)(d * a.inverse));
}

template <typename T>
hipError_t launch_logprob_bwd_t(const LogprobGrad& a, hipStream_t st) {
    constexpr int E = Vec<T>::N;
    const int64_t nv = a.V / E;  // at least the whole vectors
    const bool wave = nv <= 64 * LB_U, few = nv <= LB_FEW * LB_U && a.T <= LB_FEW;
    const int64_t tr = few ? LB_FEW : wave ? 64 : LB_BLOCK;
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
        if (few && a.dentropy)
            hipLaunchKernelGGL((logprob_grad<T, LB_FEW, true>), grid, block, 0, st, b, n);
        else if (few)
            hipLaunchKernelGGL((logprob_grad<T, LB_FEW, false>), grid, block, 0, st, b, n);
        else if (wave && a.dentropy)
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

// How a batch is taken, by its rows' 16-byte vectors.  us of one call among others, f: binary32, b:
// bfloat16 with the entropy; "held w" / "stream w": a workgroup of w wavefronts a row (w = 1: four
// rows), xS: for each of S chunks.
//
// Up to 256 vectors, where there is a row for each CU: 16 lanes a row up to 64 vectors, else 32
// (short, against held 1: 32768 x 32 b 4.8 / 14.8, 100000 x 64 f 11.5 / 33.2, 32768 x 500 b 10.9 /
// 18.2, 16385 x 1000 b 10.3 / 13.1 and f 13.5 / 14.1; 1000 x 32 f 2.7 / 3.3). Up to 512: a
// wavefront a row where there are rows for all of them (8192 x 4000 b held 1 20.4, held 4 23.6;
// but 256 x 4000 b 5.5 / 4.1). Up to 2048: held 4 (256 x 8000 f 5.3, stream 4 5.3, held 4 x2 6.6).
// Beyond that streams, by eight wavefronts (256 x 16000 f stream 8 6.2, stream 4 6.9, held 8 7.0;
// 1024 x 128256 f 79.6 / 79.4 / 95; 2048 x 128256 b 84.7 / 90.6 / 105), or by four where rows are
// not long and there are more of them than CUs (400 x 32000 b stream 4 10.5, 8 10.6; 8192 x 50257
// b 139 / 153; 8192 x 16000 b 48.3 / 52.5).
//
// Few long rows are split into as many chunks as give each CU one, of at least 4096 vectors, or up
// to four in any case (64 x 128256 f stream 8 x4 10.4, x8 11.2; 16 x 128256 f x8 7.8, x6 8.2; 128
// x 65536 f x2 9.9, x1 10.5; 16 x 65536 f x4 6.9); eight rows and fewer into up to 64 of at
// least 512 vectors (1 x 128256 f held 4 x32 5.2, x16 5.7; 1 x 50257 f x32 4.9, x8 5.5).
//
// With alternatives (5 of them) rows are held by eight wavefronts from 2048 vectors on (16 x 16000
// f held 8 7.2, held 4 7.5; but 4096 x 16000 f 50.9 / 47.1), beyond 8192 vectors in chunks that
// four hold, of about 2048 where rows are few (64 x 128256 b x8 14.2, x4 15.0).  Batches of 3 rows
// for 2 CUs and more are streamed from 4096 vectors on (held / stream 4: 512 x 25000 f 16.0 /
// 15.4, 4096 x 50000 b 102 / 83, 1024 x 128256 f 105 / 84, 2048 x 128256 b 125 / 93; but 256 x
// 50000 b 13.5 / 14.0, 4096 x 16000 f 49.1 / 51.2), of a row a CU from 8192 on, in two chunks from
// 16384 on (256 x 100000 b 22.8 / 20.2, 256 x 256512 b 39.8 / 33.8): up to 32 alternatives, which
// the maxima of 64 lanes bound well (1024 x 128256 b top-20 72 / 54, top-50 76 / 86).
LogprobPlan logprob_plan(int64_t N, int64_t V, int K, int dtype, int cus) {
    const int64_t E = dtype == 1 ? 8 : 4, c = cus;
    const int64_t nv = (V + E - 1) / E;
    const int64_t hold4 = 256 * 16, hold8 = 512 * 16;  // vectors
    LogprobPlan p{4, 1, V, N, 0, 0};
    int64_t S = 1;
    if (K > 0 && K <= 32 && ((nv > hold8 && N >= c) || (nv > hold4 && 2 * N >= 3 * c))) {
        p.stream = 4;
        S = 2 * N < 3 * c && nv >= 2 * hold8 ? 2 : 1;
    } else if (nv > 4096 && N <= 8) {
        const int64_t most = K > 16 ? 32 : 64;
        S = nv / 512 < most ? nv / 512 : most;
    } else if (K == 0 && nv > 4096 && N < c) {
        const int64_t most = nv / 4096 > 4 ? nv / 4096 : 4;
        S = c / N < most ? c / N : most;
    } else if (K > 0 && nv > hold8) {
        const int64_t want = 2 * c / N, most = nv / 2048;
        S = want < most ? want : most;
    }
    // chunks that the registers hold, where they have to
    if (K > 0 && !p.stream && nv > hold8 && S < (nv + hold4 - 1) / hold4)
        S = (nv + hold4 - 1) / hold4;
    const int64_t vecs = (nv + S - 1) / S;
    if (p.stream) {
        // (streamed with alternatives)
    } else if (K == 0 && vecs > 2048) {
        p.stream = nv <= hold8 && 2 * N >= 3 * c ? 4 : 8;
    } else if (S == 1) {
        p.W = nv <= 512 && N >= 4 * c ? 1
              : nv <= 2048 || (nv <= hold4 && N >= 8 * c) ? 4 : 8;
    }
    if (K == 0 && nv <= 256 && N >= c) p.lanes = nv <= 64 ? 16 : 32;
    if (S > 1) {
        p.chunk = vecs * E;
        S = (V + p.chunk - 1) / p.chunk;
    }
    p.S = (int)S;
    // 2^16 chunks a launch, or one row; 2^22 rows (a launch has fewer than 2^32 threads)
    const int64_t rows = S > 1 ? ((int64_t)1 << 16) / S : (int64_t)1 << 22;
    p.rows = rows < 1 ? 1 : rows < N ? rows : N;
    return p;
}

}  // namespace osm
