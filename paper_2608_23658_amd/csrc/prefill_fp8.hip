// Chunked prefill over a cache in 8 bits with plain scores (prefill_tile_fp8.hpp has the
// kernel).

#include "prefill_tile_fp8.hpp"

namespace kvattn {

hipError_t launch_prefill_fp8(const PrefillArgs& a, const PrefillLaunch& l) {
  return dispatch_prefill_fp8(a, l, PlainScore{a.scale * kLog2e});
}

}  // namespace kvattn
