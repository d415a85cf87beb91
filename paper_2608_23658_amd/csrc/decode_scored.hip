// Decode with scores that are capped, biased by distance or cut to a window: the walks of
// decode, with scores made by ModScore.
//
// What a window leaves out is never read: a sequence is walked from the block of its
// window's first token, through a block table that begins there, so that splits, merge and
// workspace are those of a context of the window's length; of that block's tokens those before
// the window are masked, and their V zeroed, in a wavefront's first step alone. A bias is one
// multiply-add a score, a cap an exponential and a reciprocal: 2 or 3% of a large batch, which
// the loads bound, and of a small one what its last step's latency grows by. In
// bf16 and over 8 bits one kernel asks what there is to do, once a step for a lane's 16 scores
// and by scalar branches; asking for each block's four by vector branches, and waiting for the
// slopes before the first step's loads, cost 0.5 us of one sequence's call (13.7 -> 13.1 with a
// cap). Per call, plain decode / window of 1024 / bias / cap / cap and bias
// (32 query heads over 8, head_dim 128, graph replay):
//   1 sequence of 3971                      11.2 / 12.9 / 12.7 / 13.3 / 13.5 us
//   12 of 1 to 4096, 64 over 8, d 64        16.7 / 11.3 / 18.6 / 19.1 / 19.4 us
//   256 of 512 to 4096                       370 /  174 /  380 /  376 /  376 us
//   6 of 700 to 131071, 8 bits              81.8 / 12.9 / 85.6 / 86.2 / 86.4 us
//   256 of 512 to 4096, fp32, d 64           364 /  173 /  375 /  370 /  371 us
//   12 of 1 to 4096, fp32, d 64             31.0 / 21.7 / 31.4 / 31.5 / 31.5 us
//   200 of 200, fp32, d 64                  33.5 / 35.4 / 35.0 / 35.3 / 36.5 us
// (in the last, plain decode's workgroups take turns, for which fp32's walk with other scores
// has no scalar registers.)

#include "decode_split.hpp"

namespace kvattn {

hipError_t launch_decode_scored(const DecodeArgs& a) {
  if (a.bf16) return dispatch_bf16(a, mod_score<Form::kAny>(a.scale, *a.mods));
  // with the library's tanh, fp32's walk is built with a cap and without
  return a.mods->softcap > 0.f ? dispatch_f32(a, mod_score<Form::kCap>(a.scale, *a.mods))
                               : dispatch_f32(a, mod_score<Form::kBias>(a.scale, *a.mods));
}

}  // namespace kvattn
