// Log probabilities of bf16 rows (one source per element type and selection, so that the build
// compiles them in parallel; the one with alternatives is logprob_top_bf16.hip).
#include "logprob.hpp"

namespace osm {
hipError_t launch_logprob_top_bf16(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                                  uint32_t* ctr, hipStream_t st);
hipError_t launch_logprob_bf16(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                              uint32_t* ctr, hipStream_t st) {
    return a.K > 0 ? launch_logprob_top_bf16(a, p, scratch, ctr, st)
                   : launch_logprob_t<bf16_t, false>(a, p, scratch, ctr, st);
}
}  // namespace osm
