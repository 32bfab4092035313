// Log probabilities of f32 rows (one source per element type and selection, so that the build
// compiles them in parallel; the one with alternatives is logprob_top_f32.hip).
#include "logprob.hpp"

namespace osm {
hipError_t launch_logprob_top_f32(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                                  uint32_t* ctr, hipStream_t st);
hipError_t launch_logprob_f32(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                              uint32_t* ctr, hipStream_t st) {
    return a.K > 0 ? launch_logprob_top_f32(a, p, scratch, ctr, st)
                   : launch_logprob_t<float, false>(a, p, scratch, ctr, st);
}
}  // namespace osm
