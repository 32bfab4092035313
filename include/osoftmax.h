/*
 * osoftmax -- row-wise softmax with the online normalizer, fused softmax +
 * top-k, sampling, log probabilities, expert routing and their gradients, for
 * AMD Instinct MI355X (gfx950).
 *
 * Method: M. Milakov and N. Gimelshein, "Online normalizer calculation for
 * softmax" (arXiv:1805.02867, 2018).
 *
 * Conventions shared by every entry point:
 *  - Buffers are device pointers on the current HIP device, owned by the
 *    caller.  Batches are row-major N x V, rows contiguous (row r starts V
 *    elements after row r-1, or ldx where an entry point has it), each pointer
 *    aligned to its element size.
 *  - Element types (dtype): OSM_F32 = IEEE binary32, OSM_BF16 = bfloat16
 *    (16-bit patterns).  Arithmetic is binary32 unless an entry point says
 *    otherwise; bfloat16 inputs are widened exactly and bfloat16 outputs are
 *    rounded to nearest even.
 *  - Calls are asynchronous: they validate the arguments on the host, enqueue
 *    work on `stream` (NULL = the default stream) and return.  A status other
 *    than OSM_OK means nothing was enqueued, except OSM_EHIP, which reports a
 *    HIP error raised while enqueuing.  Kernel faults surface on the next
 *    synchronising HIP call, as with any HIP kernel.
 *  - N = 0 is a no-op returning OSM_OK.  Sizes must satisfy 1 <= V <= 2^31-1,
 *    0 <= N <= 2^31-1.
 *  - Input and output buffers must not overlap (OSM_EINVAL otherwise).
 *  - Results are deterministic: the same call on the same device gives the
 *    same bits (fixed reduction orders, no floating-point atomics).
 *  - Non-finite inputs: -inf elements give 0 when the row has a finite
 *    element; a row holding NaN or +inf, or only -inf, gives NaN outputs
 *    (IEEE evaluation of the safe formula, Eq. 2).  Finite inputs must stay
 *    below 2.35e38 (x * log2(e) must be finite).  Top-k of a NaN row is
 *    unspecified.
 *  - Thread safety: calls may be made concurrently from several host threads
 *    and streams, including several threads on one stream.  The shared state
 *    is a per-device cache of device properties, a per-device stream-ordered
 *    memory pool, and the scratch of the split kernels, kept per stream (up
 *    to 64 streams per device; further streams get a buffer per call).  A
 *    call that uses its stream's scratch holds a per-device lock from taking
 *    the buffer until its last kernel is enqueued, so calls on one stream
 *    never interleave their kernels on shared buffers.  A stream's buffer
 *    grows in stream order and is kept until osm_stream_release(stream) or
 *    the end of the process: call osm_stream_release before destroying a
 *    stream that has used the library, so that a later stream given the same
 *    handle starts without a buffer.
 *  - Graph capture: the row kernels allocate nothing; the split kernels
 *    (small batches of long rows) allocate their stream's scratch on its
 *    first use and when it must grow.  Under HIP graph capture, either call
 *    once outside the capture on the same stream with the largest shape to
 *    be captured (the buffer is then reused and nothing is allocated), or use
 *    softmax_topk_ex_noalloc for the top-k and softmax_sample_ws,
 *    logprob_fwd_ws and balance_fwd_ws for those: an allocation recorded into
 *    a graph would leave the stream's buffer owned by the graph.
 */
#ifndef OSOFTMAX_H
#define OSOFTMAX_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#if defined(__GNUC__) || defined(__clang__)
#define OSM_API __attribute__((visibility("default")))
#else
#define OSM_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
enum osm_dtype { OSM_F32 = 0, OSM_BF16 = 1 };

/* Normalizer algorithms (Section 2 and 3 of the paper):
 *  OSM_NAIVE : Alg. 1 -- d = sum_j e^{x_j}, y_i = e^{x_i}/d.  Two loads and
 *              one store per element.  Overflows (NaN/inf outputs) once
 *              e^{x} exceeds binary32 range, x > ~88.7, as the paper warns.
 *  OSM_SAFE  : Alg. 2 -- max pass, normalizer pass, output pass.  Three
 *              loads and one store per element.
 *  OSM_ONLINE: Alg. 3 -- one pass carrying the running (max, normalizer)
 *              pair merged with Eq. 4, then the output pass.  Two loads and
 *              one store per element.
 *  OSM_RESIDENT: Alg. 3's pair (per lane, then merged with Eq. 4) with the
 *              row held in registers between the normalizer and the output:
 *              one load and one store per element.  Rows of at most
 *              OSM_RESIDENT_MAX_VEC whole 16-byte vectors (65536 binary32 or
 *              131072 bfloat16 elements, plus up to one partial vector at
 *              each end); longer rows give OSM_EUNSUPPORTED. */
enum osm_mode { OSM_NAIVE = 0, OSM_SAFE = 1, OSM_ONLINE = 2, OSM_RESIDENT = 3 };

/* Longest row of OSM_RESIDENT, in 16-byte vectors. */
#define OSM_RESIDENT_MAX_VEC 16384

/* Status codes. */
enum osm_status {
    OSM_OK = 0,
    OSM_EINVAL = 1,       /* invalid argument; nothing enqueued */
    OSM_EUNSUPPORTED = 2, /* valid but unsupported configuration */
    OSM_EHIP = 3,         /* HIP reported an error while enqueuing */
    OSM_ENOMEM = 4,       /* scratch allocation failed */
    OSM_ESCRATCH = 5      /* needs more than OSM_NOALLOC_SCRATCH_BYTES of
                             fixed scratch (softmax_topk_ex_noalloc) */
};

/* Kernel families for softmax_fwd_ex, softmax_topk_ex and softmax_topk_algo. */
enum osm_kernel {
    OSM_KERNEL_AUTO = 0,  /* what the plain entry points use */
    OSM_KERNEL_ROWS = 1,  /* param = lanes per row.  Softmax: 4, 8, 16, 32
                             (several rows per wavefront), 64 (a row per
                             wavefront) or 128, 256, 512, 1024 (a row per
                             workgroup).  Top-k: 64 or 128 (one or two
                             wavefronts per row) or 256 (a workgroup per row:
                             four wavefronts, or eight for rows of 4097 to
                             8192 whole 16-byte vectors, which eight hold in
                             registers). */
    OSM_KERNEL_SPLIT = 2  /* param = chunks per row S >= 1: a workgroup per
                             chunk; per-chunk normalizer pairs (and, for
                             top-k, per-chunk top-k keys) go through a
                             scratch array (stream-ordered allocation).
                             Softmax merges them in a second kernel; top-k
                             merges each row in the workgroup that completes
                             it, counted in a per-stream array of N
                             counters that is cleared once when allocated
                             and left cleared by every call (so calls on one
                             stream must not overlap, which stream order
                             guarantees) */
};

/* Softmax + top-k algorithms (Section 4, and the comparisons of Section 5.2):
 *  OSM_TOPK_ONLINE_FUSED  : Alg. 4 -- online pair and top-k in one pass, one
 *                           load per element.  What softmax_topk uses.
 *  OSM_TOPK_SAFE_FUSED    : a maximum pass, then the normalizer (with that
 *                           maximum) and top-k in one pass: two loads per
 *                           element.
 *  OSM_TOPK_SAFE_UNFUSED  : safe softmax (Alg. 2) writes y, then a separate
 *                           top-k over y: five accesses per element.
 *  OSM_TOPK_ONLINE_UNFUSED: online softmax (Alg. 3) writes y, then top-k over
 *                           y: four accesses per element.
 *  OSM_TOPK_VALUES        : top-k of x itself, no softmax (vals = x[z]).
 * The fused algorithms select on x; the unfused ones select on the stored y
 * (Eq. 5), so where distinct inputs round to equal outputs (mostly bfloat16
 * y) their ties go to the lower index among equal y. */
enum osm_topk_algo {
    OSM_TOPK_ONLINE_FUSED = 0,
    OSM_TOPK_SAFE_FUSED = 1,
    OSM_TOPK_SAFE_UNFUSED = 2,
    OSM_TOPK_ONLINE_UNFUSED = 3,
    OSM_TOPK_VALUES = 4
};

/* Largest K accepted by the top-k entry points. */
#define OSM_TOPK_KMAX 64

/* y = Softmax(x) row by row (Eq. 1, Section 2), for each of N rows of V
 * elements.  x: N*V elements of `dtype`, read only.  y: N*V elements of the
 * same dtype, written.  mode: an osm_mode.  The three modes compute the same
 * function (Theorem 1) and differ in their passes over memory.
 * Errors: OSM_EINVAL for N < 0, V < 1, sizes above the limits, null pointers
 * with N > 0, unknown dtype or mode, misaligned or overlapping buffers.
 * OSM_ENOMEM if the split-V scratch array cannot be allocated.
 * OSM_EUNSUPPORTED for OSM_RESIDENT rows longer than it holds. */
OSM_API int softmax_fwd(const void* x, void* y, int64_t N, int64_t V, int dtype, int mode,
                hipStream_t stream);

/* softmax_fwd with an explicit kernel family and parameter (osm_kernel);
 * OSM_KERNEL_AUTO ignores param.  OSM_RESIDENT accepts OSM_KERNEL_AUTO or
 * OSM_KERNEL_ROWS with param = 256, 512 or 1024 threads per row.  Results agree with softmax_fwd within the
 * library's accuracy (binary32 rounding differs with the reduction tree).
 * Errors: as softmax_fwd, plus OSM_EINVAL for an unknown kernel or a param
 * it does not accept. */
OSM_API int softmax_fwd_ex(const void* x, void* y, int64_t N, int64_t V, int dtype, int mode,
                   int kernel, int64_t param, hipStream_t stream);

/* Fused online softmax + top-k (Alg. 4, Section 4) over binary32 rows.
 * For each row: z = the K indices of the largest x (Eq. 5), larger first,
 * equal values in increasing index order (Alg. 4's strictly-less insertion);
 * vals[i] = softmax(x)[z[i]].  Reads x once; writes only N*K outputs.
 * x: N*V binary32.  vals: N*K binary32.  idx: N*K int32, 0-based.
 * Errors: OSM_EINVAL for K < 1, K > V, K > OSM_TOPK_KMAX, and the softmax_fwd
 * argument errors; vals and idx must not overlap x or each other. */
OSM_API int softmax_topk(const float* x, float* vals, int32_t* idx, int64_t N, int64_t V, int K,
                 hipStream_t stream);

/* softmax_topk for bfloat16 or binary32 rows (dtype: osm_dtype).  vals stay
 * binary32 and are computed from the exact widened inputs. */
OSM_API int softmax_topk_dt(const void* x, float* vals, int32_t* idx, int64_t N, int64_t V, int K,
                    int dtype, hipStream_t stream);

/* softmax_topk_dt with an explicit kernel: OSM_KERNEL_AUTO (what
 * softmax_topk_dt uses; param ignored), OSM_KERNEL_ROWS with param = lanes
 * per row: 64, 128 or 256 (one or two wavefronts, or a workgroup per row), or
 * OSM_KERNEL_SPLIT with param = chunks per row (clamped so that every chunk
 * starts inside the row).  Indices are identical across kernels; vals agree
 * within binary32 rounding of the reduction tree.
 * Errors: as softmax_topk_dt, plus OSM_EINVAL for another kernel or param,
 * or N * S >= 2^31 chunks; OSM_ENOMEM if the split scratch (N * S * (8K + 8)
 * bytes) or the row counters (4N bytes) cannot be allocated. */
OSM_API int softmax_topk_ex(const void* x, float* vals, int32_t* idx, int64_t N, int64_t V,
                            int K, int dtype, int kernel, int64_t param, hipStream_t stream);

/* Size of the fixed scratch array behind softmax_topk_ex_noalloc, per device. */
#define OSM_NOALLOC_SCRATCH_BYTES (1u << 20)

/* softmax_topk_ex for callers that cannot allocate device memory (code under
 * HIP graph capture, serving loops that must not call hipMalloc): the same
 * kernels and results, but nothing is allocated or freed, by the library or
 * through any allocating routine.  The split path (OSM_KERNEL_SPLIT, or the
 * plan's choice for small batches of long rows) keeps its per-chunk partials
 * (N * S * (8K + 8) bytes, rounded up to 256) and its N row counters (4N
 * bytes, cleared by a small kernel at each call) in a fixed array of
 * OSM_NOALLOC_SCRATCH_BYTES per device, held until the process ends; the row
 * kernels need no scratch.  Every call on a device shares that array, and it
 * keeps the last call's contents: calls that can overlap on one device (on
 * different streams, or from host threads on different streams) race and
 * must be ordered by the caller; calls on one stream are ordered by the
 * stream.  Arguments, results and errors as softmax_topk_ex, plus
 * OSM_ESCRATCH when the split path would need more than the array holds
 * (nothing enqueued) and OSM_EHIP if the array's device address could not
 * be obtained. */
OSM_API int softmax_topk_ex_noalloc(const void* x, float* vals, int32_t* idx, int64_t N,
                                    int64_t V, int K, int dtype, int kernel, int64_t param,
                                    hipStream_t stream);

/* Softmax + top-k by any osm_topk_algo, with an explicit kernel for the
 * top-k pass (kernel and param as in softmax_topk_ex; the two-wavefront
 * shape, param 128, exists for OSM_TOPK_ONLINE_FUSED only; the softmax pass
 * of the unfused algorithms uses what softmax_fwd uses).
 * y: N*V elements of dtype, written with the softmax for the unfused
 * algorithms (must not overlap x, vals or idx); ignored (may be NULL) by the
 * others.  vals: binary32; for the unfused algorithms and OSM_TOPK_VALUES
 * they are the selected elements of y (resp. x), widened exactly.
 * Errors: as softmax_topk_ex, plus OSM_EINVAL for an unknown algo or a
 * missing / misaligned / overlapping y where one is needed. */
OSM_API int softmax_topk_algo(const void* x, void* y, float* vals, int32_t* idx, int64_t N,
                              int64_t V, int K, int dtype, int algo, int kernel, int64_t param,
                              hipStream_t stream);

/* Top-k of the elements themselves, row by row (the top-k of Eq. 5 applied
 * to x): z = the K indices of the largest x, larger first, equal values in
 * increasing index order; vals = x[z] widened to binary32 (-0.0 is returned
 * as +0.0).  NaN elements are never selected; a row with fewer than K
 * non-NaN elements gets idx -1 and NaN vals in the missing places.
 * Errors: as softmax_topk_dt. */
OSM_API int topk_fwd(const void* x, float* vals, int32_t* idx, int64_t N, int64_t V, int K,
                     int dtype, hipStream_t stream);

/* Largest K of proj_softmax_topk. */
#define OSM_PROJ_KMAX 16

/* The projection ahead of the softmax in a language model (Section 1):
 * logits[n][v] = sum_k h[n][k] * w[v][k], on the matrix cores.
 * h: N*H bfloat16 (hidden vectors, row-major), w: V*H bfloat16 (one row per
 * vocabulary entry), both 16-byte aligned with H a multiple of 8.
 * logits: N*V binary32 (binary32 accumulation; the order of the sums is the
 * kernel's, so results match an exact dot product to within binary32
 * accumulation error).  logits must not overlap h or w.
 * Errors: OSM_EINVAL for N < 0, N > 65535 * 128, V < 1, H < 8, H > 2^20,
 * H not a multiple of 8, sizes above 2^31 - 1, null or misaligned
 * pointers. */
OSM_API int proj_fwd(const void* h, const void* w, float* logits, int64_t N, int64_t H,
                     int64_t V, hipStream_t stream);

/* The projection fused with the online softmax and top-k (the Discussion's
 * proposal): for each row n, z = the K indices of the largest logits (Eq. 5,
 * larger first, equal values in increasing index order) and vals[i] =
 * softmax(logits[n])[z[i]], without writing the logits anywhere.  Each
 * 256 x 256 tile of logits is reduced on chip to per-lane online pairs
 * (Alg. 3) and top-K lists (Alg. 4); partials are merged by Eq. 4 and the key
 * order.  h, w as in proj_fwd; vals: N*K binary32; idx: N*K int32, 0-based.
 * Selection is on the binary32 logits as computed by the kernel.
 * Errors: as proj_fwd, plus OSM_EINVAL for K < 1, K > V, K > OSM_PROJ_KMAX or
 * overlapping outputs; OSM_ENOMEM if the partials' scratch (N * 2S * (8K + 8)
 * bytes, S = vocabulary chunks) cannot be allocated. */
OSM_API int proj_softmax_topk(const void* h, const void* w, float* vals, int32_t* idx,
                              int64_t N, int64_t H, int64_t V, int K, hipStream_t stream);

/* What softmax_sample does with a batch.  Each setting is an array of N device
 * values, one a row, or, where its pointer is NULL, one value for all rows.
 *  temperature: logits are divided by it.  0, negative or NaN: the row's
 *               largest element is taken (the lowest index of equal ones).
 *  top_k      : the elements that are kept, in the order of Eq. 5.  0, negative
 *               or at least V: all.
 *  top_p      : of those, the shortest prefix in that order whose sum reaches
 *               this part of their sum, at least one.  At least 1 or NaN: all.
 *  min_p      : of those, the ones whose probability is at least this part of
 *               the largest one.  0, negative or NaN: all; more than 1 is 1. */
typedef struct osm_sample_params {
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all;
    int32_t top_k_all;
    float top_p_all;
    float min_p_all;
} osm_sample_params;

/* Samples one element of each row from the softmax of its logits, with the
 * row's random number given.  With w_j = e^{(x_j - max x) / temperature} and
 * the filters of osm_sample_params applied in the order in which they stand
 * there: idx[r] is the lowest kept index at which the running sum of w over the
 * kept elements, in index order, exceeds u[r] times their sum, and vals[r] its
 * probability among the kept elements (w / sum).  u below 0 or NaN counts as 0,
 * above 1 as 1; elements of weight 0 are never taken.  At 1, which no running sum
 * exceeds, it is the last kept index or one behind which less than 1e-13 of the sum
 * (with filters, than the bounds below) is left.  Weights and sums are
 * binary64, so the choice is that of the formula but for numbers u within about
 * 1e-13 of a border.  With filters some sums are of weights in fixed point, in units
 * relative to the largest: then u within 2^-49 V of a border may take its
 * neighbour, and top_p within the larger of 2^-49 V and 2^-62 V^2 may keep an
 * element more or less (both are bounds of the worst row; roundings mostly
 * cancel).  The same call gives the same result.
 * A row holding NaN or +inf, or only -inf, gives idx -1 and a NaN value.
 * x: row r starts at x + r * ldx elements, ldx >= V.  u: N binary32.  vals: N
 * binary32.  idx: N int32.  params NULL: temperature 1, no filter.
 * Errors: OSM_EINVAL for bad sizes, ldx < V, unknown dtype, null (with N > 0),
 * misaligned or overlapping buffers (the memory between rows is part of x). */
OSM_API int softmax_sample(const void* x, int64_t ldx, const float* u,
                           const osm_sample_params* params, float* vals, int32_t* idx, int64_t N,
                           int64_t V, int dtype, hipStream_t stream);

/* softmax_sample with the caller's workspace instead of the library's scratch: nothing
 * is allocated, and calls share nothing but what the caller lets them share.  For
 * HIP graph capture: graphs captured with workspaces of their own may be replayed
 * at the same time.  workspace: osm_sample_workspace(N, V, dtype) bytes, aligned
 * to 256, of any contents; NULL where that is 0.
 * Errors: as softmax_sample, OSM_EINVAL for a misaligned or overlapping workspace,
 * OSM_ESCRATCH for one that is too small. */
OSM_API int softmax_sample_ws(const void* x, int64_t ldx, const float* u,
                              const osm_sample_params* params, float* vals, int32_t* idx,
                              int64_t N, int64_t V, int dtype, void* workspace,
                              size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace that softmax_sample_ws needs for this shape on the current device
 * (0 for rows that one workgroup takes), for any ldx, alignment and settings.
 * Errors: OSM_EINVAL for bad sizes or dtype or NULL bytes. */
OSM_API int osm_sample_workspace(int64_t N, int64_t V, int dtype, size_t* bytes);

/* Largest number of experts, and of groups of them, of route_fwd. */
#define OSM_ROUTE_EMAX 1024
#define OSM_ROUTE_GMAX 64

/* Scores of a router. */
enum osm_score { OSM_SCORE_SOFTMAX = 0, OSM_SCORE_SIGMOID = 1 };

/* How route_fwd picks and weighs experts.
 *  score     : s = softmax(x) over the row, or s = 1 / (1 + e^-x).
 *  groups    : the E experts form this many groups of E / groups neighbours
 *              (1: no groups).  The best top_groups of them are searched: by
 *              their largest c (see route_fwd; group_top 1), or by the sum of
 *              their two largest s + bias (group_top 2; of one, if no other can
 *              be chosen).  Of equal groups the lower index is taken.
 *  renorm    : nonzero: weights are divided by their sum.
 *  scale     : factor of the weights. */
typedef struct osm_route {
    int score;
    int groups;
    int top_groups;
    int group_top;
    int renorm;
    float scale;
} osm_route;

/* Routes each of N tokens to K of E experts.  With s the scores and c = s + bias
 * (c = x without a bias: both scores increase with x), idx[r] are the K experts
 * of the kept groups with the largest c, larger first, equal ones in increasing
 * index order, and vals[r] = scale * s (divided by the K scores' sum with
 * renorm).  The bias takes part in the choice only.  Scores and their sums with
 * the bias are binary64.
 * An expert whose logit or bias is -inf, or whose bias is NaN, is never chosen;
 * where too few are left, the missing places get idx -1 and weight 0.  A row
 * holding NaN or +inf gives idx -1 and NaN weights.
 * x: N*E logits of dtype.  bias: E binary32 or NULL.  vals: N*K binary32.  idx:
 * N*K int32.
 * Errors: OSM_EINVAL for N < 0, E < 1, E > OSM_ROUTE_EMAX, K < 1, K > OSM_TOPK_KMAX,
 * unknown dtype or score, groups < 1, above OSM_ROUTE_GMAX or not dividing E,
 * top_groups outside [1, groups], K > top_groups * E / groups, group_top other
 * than 1 and 2, null r or (with N > 0) buffers, misaligned or overlapping
 * buffers. */
OSM_API int route_fwd(const void* x, const float* bias, float* vals, int32_t* idx, int64_t N,
                      int64_t E, int K, int dtype, const osm_route* r, hipStream_t stream);

/* The gradient of route_fwd's weights with respect to the logits: dx = sum over
 * the places i of dvals[i] * d vals[i] / dx, with the choice idx held fixed, for
 * the same score, renorm and scale (the other members of r are not read).
 * Places whose idx is outside [0, E) take no part; a row without any other gets
 * zeros.  An index that occurs twice adds both.  Sums are binary64.
 * The gradient is NaN where a NaN (for the softmax also +inf) stands among the
 * logits that the weights depend on: those of the places with renorm, one place's
 * own for the sigmoid without it, else the whole row.  Places that all have
 * -inf get zeros with renorm.
 * x: N*E logits of dtype.  idx: N*K int32.  dvals: N*K binary32.  dx: N*E
 * elements of dtype, every one written.
 * Errors: as route_fwd, for the arguments it has. */
OSM_API int route_bwd(const void* x, const int32_t* idx, const float* dvals, void* dx, int64_t N,
                      int64_t E, int K, int dtype, const osm_route* r, hipStream_t stream);

/* Largest number of given tokens a row of logprob_fwd and logprob_bwd. */
#define OSM_LOGPROB_TMAX 64

/* What logprob_fwd is asked for.  Outputs that are NULL are not written; one of them
 * at least is asked for.
 *  tokens     : N*T given tokens, T a row; NULL where T is 0.
 *  logp       : N*T.  Not NULL where T > 0.
 *  entropy    : N, or NULL.
 *  stats      : N*2, or NULL: what logprob_bwd takes.
 *  top_logp   : N*K, top_idx: N*K.  Not NULL where K > 0.
 *  T, K       : 0 <= T <= OSM_LOGPROB_TMAX, 0 <= K <= OSM_TOPK_KMAX, K <= V.
 *  temperature: logits are divided by it; positive and finite. */
typedef struct osm_logprob {
    const int32_t* tokens;
    float* logp;
    float* entropy;
    float* stats;
    float* top_logp;
    int32_t* top_idx;
    int T;
    int K;
    float temperature;
} osm_logprob;

/* Log probabilities of given tokens, the entropy and the best alternatives of each
 * row's softmax.  With z = x / temperature, m = max x and
 * s = sum of e^{(x_j - m) / temperature} over all j but one that has x_j = m (the online
 * pair's d - 1, which keeps its digits where one element has all the weight):
 *   logp[i]    = (x[t_i] - m) / temperature - ln(1 + s)   for the given token t_i,
 *   entropy    = -sum_j p_j ln p_j,  p = softmax(z),
 *   stats      = (m, s),
 *   top_idx[i] = the K indices of the largest x (Eq. 5: larger first, equal values in
 *                increasing index order), top_logp[i] their log probabilities.
 * A token outside [0, V) is ignored: its logp is 0.  Elements of -inf have no weight,
 * and a log probability of -inf.  A row holding NaN or +inf, or only -inf, gives NaN
 * (0 for ignored tokens) and top_idx -1.  x is read once; sums are binary32 (weights
 * below 2^-126 are 0 in them), the outputs are formed from them in binary64; a log
 * probability below binary32's lowest value is -inf.  Finite elements may have any size (the
 * weight of one that is more than 3.4e38 below m may count as 0, which it is but at temperatures
 * above 1e36).
 * x: row r starts at x + r * ldx elements, ldx >= V.
 * Errors: OSM_EINVAL for bad sizes, ldx < V, unknown dtype, NULL p, T, K or temperature
 * outside of what osm_logprob says, no output, null (with N > 0), misaligned or
 * overlapping buffers (the memory between rows is part of x). */
OSM_API int logprob_fwd(const void* x, int64_t ldx, const osm_logprob* p, int64_t N, int64_t V,
                        int dtype, hipStream_t stream);

/* logprob_fwd with the caller's workspace instead of the library's scratch (as
 * softmax_sample_ws): osm_logprob_workspace(N, V, K, dtype) bytes, aligned to 256, of any
 * contents; NULL where that is 0.
 * Errors: as logprob_fwd, OSM_EINVAL for a misaligned or overlapping workspace,
 * OSM_ESCRATCH for one that is too small. */
OSM_API int logprob_fwd_ws(const void* x, int64_t ldx, const osm_logprob* p, int64_t N, int64_t V,
                           int dtype, void* workspace, size_t workspace_bytes,
                           hipStream_t stream);

/* Bytes of workspace that logprob_fwd_ws needs for this shape on the current device (0 for
 * rows that one workgroup takes), for any ldx, alignment, T and outputs.
 * Errors: OSM_EINVAL for bad sizes, K or dtype or NULL bytes. */
OSM_API int osm_logprob_workspace(int64_t N, int64_t V, int K, int dtype, size_t* bytes);

/* The gradient of logprob_fwd's logp and entropy with respect to the logits: with
 * p = softmax(x / temperature), g the gradients dlogp of the row's tokens inside [0, V),
 * G their sum, H the entropy and h its gradient dentropy,
 *   dx_j = (sum of g_i over t_i = j  -  p_j G  -  h p_j (ln p_j + H)) / temperature.
 * A token that occurs twice adds both; an element of -inf takes part with p_j = 0.  A row
 * whose g are all 0 (or that has no token inside) and whose h is 0 gets zeros, whatever it
 * holds; any other row with NaN stats (or h, or one of g) gets NaN.  The gradient of
 * top_logp is that of the same indices given as tokens.
 * x, ldx, tokens, T, temperature: as in logprob_fwd.  stats: N*2 and entropy: N, as
 * logprob_fwd wrote them for this x and temperature (entropy is read with dentropy only, and
 * may be NULL without it).  dlogp: N*T, NULL where T is 0.  dentropy: N, or NULL (0).  dx: row r at dx + r * lddx
 * elements of dtype, lddx >= V, every element of the rows written, none between them.
 * Errors: OSM_EINVAL for bad sizes, ldx or lddx < V, unknown dtype, bad T or temperature,
 * neither dlogp nor dentropy, null (with N > 0), misaligned or overlapping buffers. */
OSM_API int logprob_bwd(const void* x, int64_t ldx, const int32_t* tokens, const float* stats,
                        const float* entropy, const float* dlogp, const float* dentropy, void* dx,
                        int64_t lddx, int64_t N, int64_t V, int T, int dtype, float temperature,
                        hipStream_t stream);

/* The loss that keeps a router's experts in use, for each of S sequences of tokens packed one
 * behind the other: sequence i is rows starts[i] to starts[i + 1] - 1 of the batch, all of it
 * with starts NULL and S 1.  With q the shares of a row's experts (OSM_SCORE_SOFTMAX: the
 * softmax; OSM_SCORE_SIGMOID: 1 / (1 + e^-x) over its sum), over the n rows of the sequence
 * that take part:
 *   rows      = n,
 *   counts[e] = how often e stands among their K indices,
 *   probs[e]  = the mean of q_e,
 *   loss      = scale * E / (K n) * sum_e counts[e] probs[e]  (scale for even counts).
 * A row takes part if one of its indices is in [0, E); others, such as the -1 that
 * route_fwd gives where it chooses none, are not counted.  So padding is a row of -1, or
 * a row before starts[0] or from starts[S] on.  An index that occurs twice counts twice.  n = 0
 * gives zeros.  A row that takes part and whose shares are no numbers (a NaN, only -inf, for
 * the softmax +inf) makes its sequence's probs and loss NaN.  Finite logits may have any size.
 * x: N*E logits of dtype.  idx: N*K int32, as route_fwd gave them.  starts: S + 1 int32 that do
 * not decrease, or NULL; numbers outside [0, N] are taken as the nearest inside, results for
 * decreasing ones are unspecified.  loss: S binary32.  counts: S*E int32.  probs: S*E
 * binary32.  rows: S int32.  Shares are binary32; those below 2^-126 (OSM_SCORE_SIGMOID:
 * 2^-66) may be 0.  Sums over rows are binary64 but for up to 64 rows of a team of lanes and up
 * to 8 teams, which are added in binary32; of a sequence longer than a workgroup's rows, each
 * workgroup's sum is rounded to binary32 once.  N = 0 is no no-op here: the outputs are zeros.
 * Errors: OSM_EINVAL for N < 0, E < 1, E > OSM_ROUTE_EMAX, K < 1, K > OSM_TOPK_KMAX, S < 1,
 * N * K, S or S * E above 2^31 - 1, starts NULL with S > 1, unknown dtype or score, null
 * (x and idx only with N > 0), misaligned or overlapping buffers; OSM_ENOMEM if the
 * scratch cannot be allocated. */
OSM_API int balance_fwd(const void* x, const int32_t* idx, const int32_t* starts, float* loss,
                        int32_t* counts, float* probs, int32_t* rows, int64_t N, int64_t E, int K,
                        int64_t S, int dtype, int score, float scale, hipStream_t stream);

/* balance_fwd with the caller's workspace instead of the library's scratch (as
 * softmax_sample_ws): osm_balance_workspace(N, E, S) bytes, aligned to 256, of any contents;
 * NULL where that is 0.
 * Errors: as balance_fwd, OSM_EINVAL for a misaligned or overlapping workspace, OSM_ESCRATCH
 * for one that is too small. */
OSM_API int balance_fwd_ws(const void* x, const int32_t* idx, const int32_t* starts, float* loss,
                           int32_t* counts, float* probs, int32_t* rows, int64_t N, int64_t E,
                           int K, int64_t S, int dtype, int score, float scale, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace that balance_fwd_ws needs for this shape on the current device.
 * Errors: OSM_EINVAL for bad sizes or NULL bytes. */
OSM_API int osm_balance_workspace(int64_t N, int64_t E, int64_t S, size_t* bytes);

/* The gradient of balance_fwd's loss with respect to the logits, through the shares (the
 * counts have none): for a row that takes part in a sequence,
 *   dx_j = dloss * scale * E / (K n^2) * q_j (counts[j] - sum_e counts[e] q_e),
 * for the sigmoid times 1 - 1 / (1 + e^-x_j); zeros for every other row.
 * counts: S*E and rows: S as balance_fwd gave them, or summed over all the ranks that share
 * the loss.  dloss: S binary32.  dx: N*E elements of dtype, every one written.  The others: as
 * in balance_fwd.  N = 0 is a no-op.
 * Errors: as balance_fwd, for the arguments it has. */
OSM_API int balance_bwd(const void* x, const int32_t* idx, const int32_t* starts,
                        const int32_t* counts, const int32_t* rows, const float* dloss, void* dx,
                        int64_t N, int64_t E, int K, int64_t S, int dtype, int score, float scale,
                        hipStream_t stream);

/* Reference streaming kernels, for measurement only (nothing of the method):
 * op 0 reads `bytes` bytes of x (y: a device buffer of at least 1 KB that
 * the kernel may write, as a sink the compiler cannot remove); op 1 copies
 * `bytes` bytes of x to y, with 16-byte non-temporal accesses: the
 * plain read and copy rates against which the other kernels' bandwidth is
 * judged.  x and y 16-byte aligned, bytes a multiple of 16, x and y not
 * overlapping (op 1).  Each wavefront streams one contiguous span.
 * Errors: OSM_EINVAL for another op, bytes < 0 or not
 * a multiple of 16, null or misaligned pointers, overlap. */
OSM_API int osm_ref_stream(int op, const void* x, void* y, int64_t bytes, hipStream_t stream);

/* Releases the scratch buffers the library keeps for `stream` (split
 * kernels' partials and row counters): they are freed in stream order, behind
 * the work already enqueued on the stream, which still completes normally;
 * the next call on the stream allocates afresh.  Call it before destroying a
 * stream that has used the library.  A stream without buffers is a no-op.
 * Errors: OSM_EHIP if HIP rejects the stream-ordered free (for example a
 * stream already destroyed). */
OSM_API int osm_stream_release(hipStream_t stream);

/* Kernel family and parameter softmax_fwd would use for this shape on the
 * current device, with x and y congruent modulo 16 bytes (for OSM_RESIDENT:
 * OSM_KERNEL_ROWS and the threads per row; for N = 0, which launches nothing,
 * those of one row).  Errors: OSM_EINVAL
 * for bad sizes, dtype or null outputs; OSM_EUNSUPPORTED for OSM_RESIDENT
 * rows it cannot hold. */
OSM_API int osm_plan(int64_t N, int64_t V, int dtype, int mode, int* kernel, int64_t* param);

/* Kernel family and parameter the top-k entry points would use for this
 * shape on the current device (for N = 0 those of one row).  Errors: OSM_EINVAL for bad sizes, dtype, K
 * or null outputs. */
OSM_API int osm_topk_plan(int64_t N, int64_t V, int dtype, int K, int* kernel, int64_t* param);

/* Static description of a status code (never NULL). */
OSM_API const char* osm_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* OSOFTMAX_H */
