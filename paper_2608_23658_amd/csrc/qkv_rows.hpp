// Norm and rotation of a run of q or k rows, held by one wavefront in the order in which
// the cache's K tile has them.
//
// A wavefront has one head's rows of 16 consecutive tokens: lane l has token l % 16 and,
// of its row's 16-byte chunks, chunk 4 i + l / 16 in register i. So a register's 64 lanes
// are 1 KiB of a K tile as it lies in the cache; a row's sum is a lane's own and one
// exchange between the four lanes of a row; and the two dims of a pair, half the rotated
// dims apart, are a whole number of registers apart in the same lane (32 rotated dims of
// bf16 excepted: there they are two lanes of a row).
#pragma once

#include "common.hpp"
#include "launch.hpp"

namespace kvattn {

// kRot: registers of rotated chunks (0: no rotation). kEven: pairs are adjacent dims.
template <int ESZ, int D, int kRot, bool kEven>
struct QkvRows {
  static constexpr int kVec = 16 / ESZ;            // elements per chunk
  static constexpr int kN = D / kVec / 4;          // chunks per lane
  static constexpr int kElems = kN * kVec;
  static constexpr int kRotDim = kRot * 4 * kVec;
  static constexpr bool kSwap = kRot == 1 && !kEven;   // a pair is in two lanes
  static constexpr int kPairs = kSwap ? kVec : kRot * kVec / 2;   // cosines per lane
  static constexpr int kRun = kEven && kRot ? kVec / 2 : kVec;    // of them in a row of the table
  static_assert(kRot <= kN && (kRot % 2 == 0 || kRot == 1), "whole registers");

  float cs[kPairs ? kPairs : 1], sn[kPairs ? kPairs : 1];
  float w[kElems];   // the norm's weight

  static __device__ __forceinline__ int row() { return threadIdx.x % kWave / 16; }

  // First pair of the lane's i-th run of kRun pairs.
  static __device__ __forceinline__ int first_pair(int i) {
    return kSwap ? row() % 2 * kVec : (4 * i + row()) * kRun;
  }

  // The cosines and sines of token t's positions. A position outside the table gives NaN.
  __device__ __forceinline__ void load_turns(const QkvArgs& a, int t) {
    if constexpr (kRot > 0) {
      constexpr int kHalf = kRotDim / 2;
      const bool one = a.axis_end[0] >= kHalf;
#pragma unroll
      for (int i = 0; i < kPairs / kRun; ++i) {
        const int p0 = first_pair(i);
        float* c = cs + i * kRun;
        float* s = sn + i * kRun;
        if (one) {
          const int pos = a.positions[t];
          const bool in = (unsigned)pos < (unsigned)a.table_len;
          const float* at = a.table + (size_t)(in ? pos : 0) * kRotDim + p0;
          load_run(at, c);
          load_run(at + kHalf, s);
          if (!in) {
#pragma unroll
            for (int e = 0; e < kRun; ++e) c[e] = s[e] = NAN;
          }
        } else {
#pragma unroll
          for (int e = 0; e < kRun; ++e) {
            const int p = p0 + e;
            const int axis = (p >= a.axis_end[0]) + (p >= a.axis_end[1]) + (p >= a.axis_end[2]);
            const int pos = a.positions[(size_t)axis * a.num_tokens + t];
            const bool in = (unsigned)pos < (unsigned)a.table_len;
            const float* at = a.table + (size_t)(in ? pos : 0) * kRotDim + p;
            c[e] = in ? at[0] : NAN;
            s[e] = in ? at[kHalf] : NAN;
          }
        }
      }
    }
  }

  static __device__ __forceinline__ void load_run(const float* at, float* to) {
    if constexpr (kRun % 4 == 0) {
#pragma unroll
      for (int e = 0; e < kRun; e += 4) {
        const float4 v = *reinterpret_cast<const float4*>(at + e);
        to[e] = v.x;
        to[e + 1] = v.y;
        to[e + 2] = v.z;
        to[e + 3] = v.w;
      }
    } else {
      const float2 v = *reinterpret_cast<const float2*>(at);
      to[0] = v.x;
      to[1] = v.y;
    }
  }

  static __device__ __forceinline__ void widen(uint4 v, float* x) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (ESZ == 2) {
        x[2 * e] = bf16lo(u[e]);
        x[2 * e + 1] = bf16hi(u[e]);
      } else {
        x[e] = __uint_as_float(u[e]);
      }
    }
  }
  // Rounds to nearest even, the only rounding of a row's values.
  static __device__ __forceinline__ uint4 narrow(const float* x) {
    if constexpr (ESZ == 2)
      return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                        pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    else
      return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                        __float_as_uint(x[3]));
  }

  __device__ __forceinline__ void load_weight(const uint8_t* weight) {
    if (!weight) return;
#pragma unroll
    for (int i = 0; i < kN; ++i)
      widen(reinterpret_cast<const uint4*>(weight)[4 * i + row()], w + i * kVec);
  }

  // x * rsqrt(mean(x^2) + eps) * w, in fp32
  __device__ __forceinline__ void norm(float (&x)[kElems], float eps) const {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kElems; ++e) sum = fmaf(x[e], x[e], sum);
    const float by = rsqrtf(fmaf(cross_row_sum(sum), 1.f / D, eps));
#pragma unroll
    for (int e = 0; e < kElems; ++e) x[e] = x[e] * by * w[e];
  }

  __device__ __forceinline__ void rotate(float (&x)[kElems]) const {
    if constexpr (kSwap) {
      const bool second = row() >= 2;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float other = __shfl_xor(x[e], 32, kWave);
        x[e] = fmaf(x[e], cs[e], second ? other * sn[e] : -other * sn[e]);
      }
    } else if constexpr (kEven) {
#pragma unroll
      for (int p = 0; p < kPairs; ++p) turn(x[2 * p], x[2 * p + 1], cs[p], sn[p]);
    } else {
#pragma unroll
      for (int p = 0; p < kPairs; ++p) turn(x[p], x[p + kPairs], cs[p], sn[p]);
    }
  }
  static __device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float a1 = fmaf(a, c, -(b * s));
    b = fmaf(b, c, a * s);
    a = a1;
  }
};

}  // namespace kvattn
