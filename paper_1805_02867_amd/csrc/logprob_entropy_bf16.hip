// Log probabilities of bf16 rows with the entropy.
#include "logprob.hpp"

namespace osm {
hipError_t launch_logprob_entropy_bf16(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                                       uint32_t* ctr, hipStream_t st) {
    return launch_logprob_t<bf16_t, false, true>(a, p, scratch, ctr, st);
}
}  // namespace osm
