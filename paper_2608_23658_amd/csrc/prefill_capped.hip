// Chunked prefill with capped scores.

#include "prefill_scored.hpp"

namespace kvattn {

hipError_t launch_prefill_capped(const PrefillArgs& a, const PrefillLaunch& l) {
  return dispatch_prefill_scored<Form::kCap>(a, l);
}

}  // namespace kvattn
