// Decode with scores that are capped, biased by distance or cut to a window.

#include "decode_split.hpp"

namespace kvattn {

hipError_t launch_decode_scored(const DecodeArgs& a) {
  return dispatch_decode(a, mod_score(a.scale, *a.mods));
}

}  // namespace kvattn
