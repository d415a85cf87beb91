// Decode with scores that are capped, biased by distance or cut to a window.

#include "decode_split.hpp"

namespace kvattn {

hipError_t launch_decode_scored(const DecodeArgs& a) {
  if (a.bf16) return dispatch_bf16(a, mod_score<Form::kAny>(a.scale, *a.mods));
  // with the library's tanh, fp32's walk is built with a cap and without
  return a.mods->softcap > 0.f ? dispatch_f32(a, mod_score<Form::kCap>(a.scale, *a.mods))
                               : dispatch_f32(a, mod_score<Form::kBias>(a.scale, *a.mods));
}

}  // namespace kvattn
