// The norm, rotation and cache write of qkv_append.hip over a cache in 8 bits: K rows
// are scaled and rounded from the fp32 values that the rotation gives. One launch: the
// first workgroups append K and V as append_fp8.hpp does, the others have the q rows. A K
// row is normed and rotated in the lanes that hold it for its scale.
// 8192 tokens in order, 32 query heads over 8 of 128, bf16, inputs not in a cache: 53.5 us, where
// copying as many bytes takes 38.5; 4096 tokens of 64 over 8: 39.5, copy 32.9, and 35.1 in calls
// one after another. With K's pairs looked up value by value it was 93.8 and 73.6. 256 scattered tokens: 16.2 us
// (25.4), a chain of latencies: slots, exponents and positions, rows and table, codes.

#include "append_fp8.hpp"
#include "launch.hpp"
#include "qkv_rows.hpp"

namespace kvattn {

// Norm and rotation of K rows as append_fp8 holds them, along the lanes.
template <int ESZ, int D, int kRotDim, bool kEven>
struct KeyPrep {
  static constexpr bool kOn = true;
  using R = LaneRows<ESZ, D, kRotDim, kEven, false>;
  const QkvArgs& a;

  // The lane's pieces x of token t, the first of them the row's piece-th.
  __device__ __forceinline__ void apply(float* x, int t, int piece) const {
    float c[R::kPairs], s[R::kPairs], w[R::kElems];
    R::turns(a, t, piece, c, s);
    if (a.k_weight) {
      R::weights(a.k_weight, piece, w);
      R::norm(x, w, a.eps);
    }
    R::rotate(x, piece, c, s);
  }
};

template <int ESZ, int D, int kRotDim, bool kEven, int kWin>
__global__ __launch_bounds__(kQkvWaves * kWave) void qkv_append_fp8_kernel(QkvArgs a,
                                                                           int append_wgs,
                                                                           int groups,
                                                                           int per_wave) {
  static_assert(kQkvWaves == kAppendWaves, "one launch");
  if ((int)blockIdx.x < append_wgs)
    append_fp8<ESZ, D, kWin>(blockIdx.x, a.k, a.k_stride, a.v, a.v_stride, a.slot_mapping, a.kv,
                             a.num_tokens, a.num_kv_heads, a.num_blocks * kBS,
                             KeyPrep<ESZ, D, kRotDim, kEven>{a});
  else
    q_rows<ESZ, D, kRotDim, kEven>(a, blockIdx.x - append_wgs, groups, per_wave);
}

template <int ESZ, int D, int kRotDim, bool kEven>
static hipError_t launch_qkv_fp8_t(const QkvArgs& a) {
  const int win = append_window(a.num_tokens);
  const long long append_wgs = ((long long)a.num_tokens + win - 1) / win * a.num_kv_heads;
  const QkvSplit rows =
      qkv_split(((long long)a.num_tokens + kRunTokens - 1) / kRunTokens, a.num_q_heads);
  const long long blocks = append_wgs + rows.workgroups;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  auto kernel = win == kFewWindow    ? qkv_append_fp8_kernel<ESZ, D, kRotDim, kEven, kFewWindow>
                : win == kSomeWindow ? qkv_append_fp8_kernel<ESZ, D, kRotDim, kEven, kSomeWindow>
                                     : qkv_append_fp8_kernel<ESZ, D, kRotDim, kEven, kWindow>;
  trace_before(a.stream, "qkv_append_fp8");
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kQkvWaves * kWave), 0, a.stream, a,
                     (int)append_wgs, rows.groups, rows.per_wave);
  trace_after(a.stream);
  return hipGetLastError();
}

template <int ESZ, int D>
static hipError_t launch_qkv_fp8_d(const QkvArgs& a) {
  return with_rotation<ESZ, D>(a, [&](auto rot, auto even) {
    return launch_qkv_fp8_t<ESZ, D, decltype(rot)::value, decltype(even)::value>(a);
  });
}

hipError_t launch_qkv_append_fp8(const QkvArgs& a) {
  if (a.head_dim == 128)
    return a.esz == 2 ? launch_qkv_fp8_d<2, 128>(a) : launch_qkv_fp8_d<4, 128>(a);
  if (a.head_dim == 64) return a.esz == 2 ? launch_qkv_fp8_d<2, 64>(a) : launch_qkv_fp8_d<4, 64>(a);
  return hipErrorNotSupported;
}

}  // namespace kvattn
