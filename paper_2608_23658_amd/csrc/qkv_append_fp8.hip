// The norm, rotation and cache write of qkv_append.hip over a cache in 8 bits: K rows
// are scaled and rounded from the fp32 values that the rotation gives. One launch: the
// first workgroups append K and V as append_fp8.hpp does, the others have the q rows.

#include "append_fp8.hpp"
#include "launch.hpp"
#include "qkv_rows.hpp"

namespace kvattn {

// Norm and rotation of K rows as append_fp8 holds them: a row's 16-byte pieces in 8 or 16
// neighbouring lanes (D elements of fp32: 32 pieces, two in each of 16 lanes).
// kRotDim 0: no rotation.
template <int ESZ, int D, int kRotDim, bool kEven>
struct KeyPrep {
  static constexpr bool kOn = true;
  static constexpr int kVec = 16 / ESZ, kCh = D / kVec;
  static constexpr int kPer = kCh > 16 ? kCh / 16 : 1;   // pieces of a row in a lane
  static constexpr int kOff = kRotDim / 2 / kVec;        // pieces between the two of a pair
  const QkvArgs& a;

  // The kPer pieces x of token t, the first of them the row's piece-th.
  __device__ __forceinline__ void apply(float* x, int t, int piece) const {
    if (a.k_weight) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kPer * kVec; ++e) sum = fmaf(x[e], x[e], sum);
      sum += dpp_mov<kDppQuadSwap1>(sum);
      sum += dpp_mov<kDppQuadSwap2>(sum);
      sum += dpp_mov<kDppRowHalfMirror>(sum);
      if constexpr (kCh > 8) sum += dpp_mov<kDppRowMirror>(sum);
      const float by = rsqrtf(fmaf(sum, 1.f / D, a.eps));
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        float w[kVec];
        QkvRows<ESZ, D, 0, false>::widen(
            reinterpret_cast<const uint4*>(a.k_weight)[piece + 16 * p], w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[p * kVec + e] = x[p * kVec + e] * by * w[e];
      }
    }
    if constexpr (kRotDim > 0) {
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        if constexpr (kEven) {
          if ((piece + 16 * p) * kVec < kRotDim) {
#pragma unroll
            for (int m = 0; m < kVec / 2; ++m) {
              const float2 cs = turn_of((piece + 16 * p) * (kVec / 2) + m, t);
              turn(x[p * kVec + 2 * m], x[p * kVec + 2 * m + 1], cs);
            }
          }
        } else if constexpr (kOff >= 16) {   // both of a pair in the lane
          if (p < kPer / 2) {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              turn(x[p * kVec + e], x[(p + kPer / 2) * kVec + e],
                   turn_of((piece + 16 * p) * kVec + e, t));
          }
        } else if (p == 0) {                 // the pair's other dim kOff lanes away
          const bool in = piece < 2 * kOff, second = piece & kOff;
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float other = __shfl_xor(x[e], kOff, kWave);
            if (in) {
              const float2 cs = turn_of(piece % kOff * kVec + e, t);
              x[e] = fmaf(x[e], cs.x, second ? other * cs.y : -other * cs.y);
            }
          }
        }
      }
    }
  }

  static __device__ __forceinline__ void turn(float& u, float& v, float2 cs) {
    QkvRows<ESZ, D, 0, false>::turn(u, v, cs.x, cs.y);
  }

  // Cosine and sine of pair p for token t; NaN for a position outside the table.
  __device__ __forceinline__ float2 turn_of(int p, int t) const {
    const int axis = (p >= a.axis_end[0]) + (p >= a.axis_end[1]) + (p >= a.axis_end[2]);
    const int pos = a.positions[(size_t)axis * a.num_tokens + t];
    const bool in = (unsigned)pos < (unsigned)a.table_len;
    const float* at = a.table + (size_t)(in ? pos : 0) * kRotDim + p;
    return in ? make_float2(at[0], at[kRotDim / 2]) : make_float2(NAN, NAN);
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
    qkv_rows<ESZ, D, kRotDim * ESZ / 64, kEven, false>(a, blockIdx.x - append_wgs, groups,
                                                       per_wave);
}

template <int ESZ, int D, int kRotDim, bool kEven>
static hipError_t launch_qkv_fp8_t(const QkvArgs& a) {
  const int win = append_window(a.num_tokens);
  const long long append_wgs = ((long long)a.num_tokens + win - 1) / win * a.num_kv_heads;
  const QkvSplit rows = qkv_split(a.num_tokens, a.num_q_heads);
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
