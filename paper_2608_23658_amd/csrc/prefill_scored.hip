// Chunked prefill with scores that are cut to a window, and the choice between them and
// biased and capped ones, which have kernels of their own.

#include "prefill_scored.hpp"

namespace kvattn {

hipError_t launch_prefill_scored(const PrefillArgs& a, const PrefillLaunch& l) {
  if (a.mods->softcap > 0.f) return launch_prefill_capped(a, l);
  if (a.mods->slopes) return launch_prefill_biased(a, l);
  return dispatch_prefill_scored<Form::kWindow>(a, l);
}

}  // namespace kvattn
