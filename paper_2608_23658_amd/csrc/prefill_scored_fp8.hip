// Chunked prefill over a cache in 8 bits with scores that are capped, biased by distance or
// cut to a window.

#include "prefill_tile_fp8.hpp"

namespace kvattn {

hipError_t launch_prefill_scored_fp8(const PrefillArgs& a, const PrefillLaunch& l) {
  return with_form(a.scale, *a.mods,
                   [&](const auto& score) { return dispatch_prefill_fp8(a, l, score); });
}

}  // namespace kvattn
