// Decode with plain scores (decode_split.hpp has the kernels), over one tensor or two.

#include "decode_split.hpp"

namespace kvattn {

hipError_t launch_decode(const DecodeArgs& a) {
  const PlainScore score = {a.scale * kLog2e};
  if (a.kv2) {   // two-tensor layer: built for bf16, head_dim 128
    if (!a.bf16 || a.head_dim != 128) return hipErrorNotSupported;
    switch (a.num_q_heads / a.num_kv_heads) {
      case 1: return launch_decode_t<128, 1, true, true, false>(a, score);
      case 2: return launch_decode_t<128, 2, true, true, false>(a, score);
      case 4: return launch_decode_t<128, 4, true, true, false>(a, score);
      case 8: return launch_decode_t<128, 8, true, true, false>(a, score);
      default: return hipErrorInvalidValue;
    }
  }
  return a.bf16 ? dispatch_bf16(a, score) : dispatch_f32(a, score);
}

}  // namespace kvattn
