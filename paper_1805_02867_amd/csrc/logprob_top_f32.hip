// Log probabilities of f32 rows with alternatives.
#include "logprob.hpp"

namespace osm {
hipError_t launch_logprob_top_f32(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                                  uint32_t* ctr, hipStream_t st) {
    return launch_logprob_t<float, true, true>(a, p, scratch, ctr, st);
}
}  // namespace osm
