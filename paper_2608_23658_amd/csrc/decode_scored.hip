// Decode with scores that are capped, biased by distance or cut to a window: the walks of
// decode, with scores made by ModScore.
//
// What a window leaves out is never read: a sequence is walked from the block of its
// window's first token, through a block table that begins there, so that splits, merge and
// workspace are those of a context of the window's length; of that block's tokens those before
// the window are masked, and their V zeroed, in a wavefront's first step alone. A bias is one
// multiply-add a score, a cap an exponential and a reciprocal: both disappear behind the loads,
// which bound a large batch, and cost a small one what its last step's latency grows by. In
// bf16 and over 8 bits one kernel asks for each score what there is to do. Per call, plain decode / window of 1024 / bias / cap / cap and bias
// (32 query heads over 8, head_dim 128, graph replay):
//   1 sequence of 3971                      11.2 / 13.1 / 13.1 / 13.6 / 14.0 us
//   12 of 1 to 4096, 64 over 8, d 64        16.5 / 12.2 / 17.8 / 18.5 / 18.8 us
//   256 of 512 to 4096                       368 /  170 /  369 /  369 /  370 us
//   6 of 700 to 131071, 8 bits              86.7 / 13.6 / 81.6 / 82.6 / 82.9 us

#include "decode_split.hpp"

namespace kvattn {

hipError_t launch_decode_scored(const DecodeArgs& a) {
  if (a.bf16) return dispatch_bf16(a, mod_score<Form::kAny>(a.scale, *a.mods));
  // with the library's tanh, fp32's walk is built with a cap and without
  return a.mods->softcap > 0.f ? dispatch_f32(a, mod_score<Form::kCap>(a.scale, *a.mods))
                               : dispatch_f32(a, mod_score<Form::kBias>(a.scale, *a.mods));
}

}  // namespace kvattn
