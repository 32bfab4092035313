// Log probabilities of bf16 rows.  The kernels are instantiated in one source each for plain ones,
// with the entropy and with alternatives (which come with the entropy), so that the build
// compiles them in parallel.
#include "logprob.hpp"

namespace osm {
hipError_t launch_logprob_entropy_bf16(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                                      uint32_t* ctr, hipStream_t st);
hipError_t launch_logprob_top_bf16(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                                  uint32_t* ctr, hipStream_t st);
hipError_t launch_logprob_bf16(const LogprobRows& a, const LogprobPlan& p, void* scratch,
                              uint32_t* ctr, hipStream_t st) {
    if (a.K > 0) return launch_logprob_top_bf16(a, p, scratch, ctr, st);
    if (a.entropy) return launch_logprob_entropy_bf16(a, p, scratch, ctr, st);
    return launch_logprob_t<bf16_t, false, false>(a, p, scratch, ctr, st);
}
}  // namespace osm
