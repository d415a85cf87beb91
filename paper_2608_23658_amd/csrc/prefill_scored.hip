// Chunked prefill with scores that are biased by distance or cut to a window, and the choice
// between them and capped ones, which have kernels of their own.

#include "prefill_scored.hpp"

namespace kvattn {

hipError_t launch_prefill_scored(const PrefillArgs& a, const PrefillLaunch& l) {
  return a.mods->softcap > 0.f ? launch_prefill_capped(a, l)
                               : dispatch_prefill_scored<Cap::kNo>(a, l);
}

}  // namespace kvattn
