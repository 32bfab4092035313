// Host-side launchers of the device kernels (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace osm {

// Row kernels: team = lanes per row (4..64 inside a wavefront, 128..1024 one
// row per workgroup).  vec: x and y rows may be read / written as 16-byte
// vectors (x and y congruent modulo 16 bytes).
hipError_t launch_softmax_rows(const void* x, void* y, int64_t N, int64_t V, int dtype,
                               int mode, int team, bool vec, hipStream_t st);

// Split-V: S chunks of `chunk` elements per row; scratch holds N * S float2.
hipError_t launch_softmax_split(const void* x, void* y, void* scratch, int64_t N, int64_t V,
                                int dtype, int mode, int64_t S, int64_t chunk, bool vec,
                                hipStream_t st);

// Row-resident online softmax: one row per workgroup of `block` threads,
// r 16-byte vectors per lane held in registers; vec: y congruent with x
// modulo 16 bytes (vector stores), else outputs stored one by one.
hipError_t launch_softmax_resident(const void* x, void* y, int64_t N, int64_t V, int dtype,
                                   int block, int r, bool vec, hipStream_t st);

// Projection (bfloat16 h: N x H, w: V x H, H a multiple of 8 and at most
// 2^20, 16-byte aligned): logits = h . w^T in binary32; cus = compute units.
hipError_t launch_proj_logits(const void* h, const void* w, float* out, int64_t N, int64_t H,
                              int64_t V, int cus, hipStream_t st);

// Projection fused with the online softmax and top-k: the kernel layout, S
// vocabulary chunks of `tiles` tiles each, and `parts` partials per (row,
// chunk), for a device with `cus` compute units.  part holds
// proj_topk_part_bytes(N, S, parts, K) bytes.
struct ProjTopkShape {
    int cfg;
    int64_t S, tiles;
    int parts;
};
ProjTopkShape proj_topk_shape(int64_t N, int64_t H, int64_t V, int K, int cus);
size_t proj_topk_part_bytes(int64_t N, int64_t S, int parts, int K);
hipError_t launch_proj_topk(const void* h, const void* w, float* vals, int32_t* idx,
                            void* part, int64_t N, int64_t H, int64_t V, int K,
                            const ProjTopkShape& p, hipStream_t st);

// Reference streaming kernels (measurement only): op 0 reads `vecs` 16-byte
// vectors of x (y: a 1 KB sink, written only for a sum never met), op 1
// copies them to y.
hipError_t launch_ref_stream(int op, const void* x, void* y, int64_t vecs, int cus,
                             hipStream_t st);

// What the top-k kernels compute next to the selection (Section 4, and the
// comparisons of Section 5.2):
//  TK_ONLINE: the online pair, one pass (Alg. 4);
//  TK_SAFE:   a maximum pass over the row first, then the normalizer with
//             that maximum held fixed, in the pass that selects (the safe
//             softmax fused with top-k: two loads per element);
//  TK_VALUES: no softmax; the outputs are the selected inputs themselves
//             (the separate top-k of the unfused comparisons).
enum TopkVar { TK_ONLINE = 0, TK_SAFE = 1, TK_VALUES = 2 };

struct TopkLaunch {
    const void* x;
    float* vals;
    int32_t* idx;
    void* part;          // split scratch (S > 1): topk_part_bytes(N, S, K) bytes
    int64_t N, V;
    int K;
    int waves_per_row;   // S <= 1: 1, 2 (TK_ONLINE only) or 4
    int64_t S, chunk;    // chunks per row and their length in elements (S > 1)
    int cus;             // compute units of the device
    hipStream_t st;
    // S > 1: N zeroed per-row counters; each row's last chunk merges the row
    // in the same kernel, and the counters are left zeroed.
    uint32_t* ctr = nullptr;
};

// Split scratch: N * S * K 64-bit keys, then N * S normalizer pairs.
inline size_t topk_part_bytes(int64_t N, int64_t S, int64_t K) {
    return (size_t)N * (size_t)S * ((size_t)K * 8 + 8);
}

hipError_t launch_topk_online_f32(const TopkLaunch& a);
hipError_t launch_topk_online_bf16(const TopkLaunch& a);
hipError_t launch_topk_safe_f32(const TopkLaunch& a);
hipError_t launch_topk_safe_bf16(const TopkLaunch& a);
hipError_t launch_topk_values_f32(const TopkLaunch& a);
hipError_t launch_topk_values_bf16(const TopkLaunch& a);

inline hipError_t launch_topk(const TopkLaunch& a, int dtype, int var) {
    const bool bf = dtype == 1;
    switch (var) {
        case TK_ONLINE: return bf ? launch_topk_online_bf16(a) : launch_topk_online_f32(a);
        case TK_SAFE: return bf ? launch_topk_safe_bf16(a) : launch_topk_safe_f32(a);
        case TK_VALUES: return bf ? launch_topk_values_bf16(a) : launch_topk_values_f32(a);
        default: return hipErrorInvalidValue;
    }
}

// Sampling: rows of V elements, row r at x + r * ld; a setting is an array of N
// or, where that is null, one value for all rows.
struct SampleRows {
    const void* x;
    const float* u;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all;
    int32_t top_k_all;
    float top_p_all, min_p_all;
    float* vals;
    int32_t* idx;
    int64_t N, V, ld;
};
// How a batch is sampled.  S = 1: a wavefront a row (R = 0), a workgroup that holds R
// vectors a lane, or one that streams the row (R < 0).  S > 1: S chunks a row,
// `rows` rows a launch; scratch of sample_scratch_bytes, and `rows` zeroed counters,
// which are left zeroed.
struct SamplePlan {
    int R, S;
    int64_t chunk, rows;
};
struct SampleSplit {
    int S;
    int64_t chunk, row0, rows;  // the launch's rows, their chunks
    int group;                  // interleaved in groups of so many
    uint64_t* parts;
    uint64_t* mass;
    uint32_t* counts;
    uint32_t* ctr;
};
bool sample_filters(const SampleRows& a);  // whether any row may have one
SamplePlan sample_plan(int64_t N, int64_t V, int64_t ld, bool aligned, int dtype, bool filters,
                       int cus);
size_t sample_scratch_bytes(const SamplePlan& p);
hipError_t launch_sample(const SampleRows& a, const SamplePlan& p, int dtype, void* scratch,
                         uint32_t* ctr, hipStream_t st);

// Routing: rows of E scores, K experts of each (see osm_route).
struct RouteRows {
    const void* x;
    const float* bias;    // E, or null
    float* vals;          // forward: written
    int32_t* idx;         // forward: written; backward: read
    const float* dvals;   // backward
    void* dx;             // backward: written
    int64_t N;
    int E, K, groups, top_groups, group_top;
    bool sigmoid, renorm;
    float scale;
    int cus;
};
hipError_t launch_route_fwd(const RouteRows& a, int dtype, hipStream_t st);
hipError_t launch_route_bwd(const RouteRows& a, int dtype, hipStream_t st);

}  // namespace osm
