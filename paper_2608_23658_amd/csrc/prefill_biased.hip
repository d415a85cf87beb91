// Chunked prefill with biased scores.

#include "prefill_scored.hpp"

namespace kvattn {

hipError_t launch_prefill_biased(const PrefillArgs& a, const PrefillLaunch& l) {
  return dispatch_prefill_scored<Form::kBias>(a, l);
}

}  // namespace kvattn
