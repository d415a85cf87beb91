// What lies between a layer's projection and its attention, in one launch: norms of the q
// and k heads, their rotation by position, and the new K and V written into their paged
// slots (the paper, Section 3, "The contiguity constraint": one tensor per layer indexed by
// block id; Section 2: blocks of fixed size).
//
// A wavefront takes a run of 16 consecutive tokens and some of the heads (q, k and v
// alike), one head after another, so that the cosines and sines of its tokens are read
// once. Every row is read once and written once.

#include "common.hpp"
#include "launch.hpp"
#include "qkv_rows.hpp"

namespace kvattn {

template <int ESZ, int D, int kRot, bool kEven>
__global__ __launch_bounds__(kQkvWaves * kWave) void qkv_append_kernel(QkvArgs a, int groups,
                                                                       int per_wave) {
  qkv_rows<ESZ, D, kRot, kEven, true>(a, blockIdx.x, groups, per_wave);
}

template <int ESZ, int D, int kRot, bool kEven>
static hipError_t launch_qkv_t(const QkvArgs& a) {
  const QkvSplit s = qkv_split(a.num_tokens, a.num_q_heads + 2 * a.num_kv_heads);
  if (s.workgroups > 0x7fffffffLL) return hipErrorInvalidValue;
  trace_before(a.stream, "qkv_append");
  hipLaunchKernelGGL((qkv_append_kernel<ESZ, D, kRot, kEven>), dim3((unsigned)s.workgroups),
                     dim3(kQkvWaves * kWave), 0, a.stream, a, s.groups, s.per_wave);
  trace_after(a.stream);
  return hipGetLastError();
}

template <int ESZ, int D>
static hipError_t launch_qkv_d(const QkvArgs& a) {
  return with_rotation<ESZ, D>(a, [&](auto rot, auto even) {
    return launch_qkv_t<ESZ, D, decltype(rot)::value * ESZ / 64, decltype(even)::value>(a);
  });
}

hipError_t launch_qkv_append(const QkvArgs& a) {
  if (a.num_tokens == 0) return hipSuccess;
  if (a.head_dim == 128) return a.esz == 2 ? launch_qkv_d<2, 128>(a) : launch_qkv_d<4, 128>(a);
  if (a.head_dim == 64) return a.esz == 2 ? launch_qkv_d<2, 64>(a) : launch_qkv_d<4, 64>(a);
  return hipErrorNotSupported;
}

}  // namespace kvattn
