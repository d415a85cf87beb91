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

#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace kvattn {

namespace {
constexpr int kRunTokens = 16;   // tokens of a run, slots of a block
constexpr int kQkvWaves = 4;
}  // namespace

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

// The work of workgroup wg, of (runs x groups of heads): per_wave heads a wavefront, of q
// and, with kCache, k and v too.
template <int ESZ, int D, int kRot, bool kEven, bool kCache>
__device__ __forceinline__ void qkv_rows(const QkvArgs& a, int wg, int groups, int per_wave) {
  using R = QkvRows<ESZ, D, kRot, kEven>;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int row = lane / 16;
  const int hq = a.num_q_heads, hkv = a.num_kv_heads;
  const int heads = kCache ? hq + 2 * hkv : hq;
  const int h0 = (wg % groups * kQkvWaves + wave) * per_wave;
  const int h1 = min(heads, h0 + per_wave);
  if (h0 >= h1) return;
  const int t = wg / groups * kRunTokens + lane % 16;
  const bool real = t < a.num_tokens;
  const int tc = min(t, a.num_tokens - 1);

  R rows;
  if (h0 < hq + hkv) rows.load_turns(a, tc);
  uint8_t* block = nullptr;    // of the token's slot; null: it has none
  int slot = 0;
  constexpr size_t kTile = (size_t)kRunTokens * D * ESZ;
  if (kCache && h1 > hq && real) {
    slot = a.slot_mapping[t];
    if ((unsigned)slot < (unsigned)(a.num_blocks * kRunTokens)) {
      block = a.kv + (size_t)(slot / kRunTokens) * (2 * (size_t)hkv * kTile);
      slot %= kRunTokens;
    }
  }

  const uint8_t* weight = nullptr;
  for (int h = h0; h < h1; ++h) {
    const bool is_q = !kCache || h < hq, is_v = kCache && h >= hq + hkv;
    const int g = is_q ? h : is_v ? h - hq - hkv : h - hq;
    const uint8_t* src = (is_q ? a.q + (size_t)tc * a.q_stride
                               : is_v ? a.v + (size_t)tc * a.v_stride
                                      : a.k + (size_t)tc * a.k_stride) +
                         (size_t)g * (D * ESZ);
    uint4 raw[R::kN];
#pragma unroll
    for (int i = 0; i < R::kN; ++i) raw[i] = reinterpret_cast<const uint4*>(src)[4 * i + row];
    if (!is_v) {
      float x[R::kElems];
#pragma unroll
      for (int i = 0; i < R::kN; ++i) R::widen(raw[i], x + i * R::kVec);
      const uint8_t* wanted = is_q ? a.q_weight : a.k_weight;
      if (wanted) {
        if (wanted != weight) rows.load_weight(wanted);
        weight = wanted;
        rows.norm(x, a.eps);
      }
      rows.rotate(x);
#pragma unroll
      for (int i = 0; i < R::kN; ++i) raw[i] = R::narrow(x + i * R::kVec);
      if (is_q) {
        if (real) {
          uint4* to = reinterpret_cast<uint4*>(a.q_out + ((size_t)t * hq + g) * (D * ESZ));
#pragma unroll
          for (int i = 0; i < R::kN; ++i) to[4 * i + row] = raw[i];
        }
      } else if (block) {
        uint4* to = reinterpret_cast<uint4*>(block + g * kTile);
#pragma unroll
        for (int i = 0; i < R::kN; ++i) to[(4 * i + row) * kRunTokens + slot] = raw[i];
      }
    } else if (block) {
      uint8_t* to = block + (hkv + g) * kTile;
#pragma unroll
      for (int i = 0; i < R::kN; ++i) {
        const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
        const int j0 = (4 * i + row) * R::kVec;
        if constexpr (ESZ == 2) {
          uint16_t* v = reinterpret_cast<uint16_t*>(to);
#pragma unroll
          for (int e = 0; e < R::kVec; ++e)
            v[(j0 + e) * kRunTokens + slot] = (uint16_t)(u[e / 2] >> (16 * (e % 2)));
        } else {
          uint32_t* v = reinterpret_cast<uint32_t*>(to);
#pragma unroll
          for (int e = 0; e < R::kVec; ++e) v[(j0 + e) * kRunTokens + slot] = u[e];
        }
      }
    }
  }
}

// How rows are dealt to wavefronts.
struct QkvSplit {
  int per_wave, groups;   // heads of a wavefront, workgroups of a run
  long long workgroups;
};
inline QkvSplit qkv_split(int tokens, int heads) {
  const long long runs = ((long long)tokens + kRunTokens - 1) / kRunTokens;
  QkvSplit s;
  s.per_wave = runs * heads > 16384 ? 4 : 1;
  s.groups = (heads + kQkvWaves * s.per_wave - 1) / (kQkvWaves * s.per_wave);
  s.workgroups = runs * s.groups;
  return s;
}

// Calls launch with a call's rotated dims and whether its pairs are adjacent, as constants.
template <int ESZ, int D, typename Launch>
hipError_t with_rotation(const QkvArgs& a, Launch launch) {
  const std::true_type even{};
  const std::false_type halves{};
  const std::integral_constant<int, 0> none{};
  const std::integral_constant<int, 32> r32{};
  const std::integral_constant<int, 64> r64{};
  if (!a.table) return launch(none, halves);
  if (a.rot == 32) return a.interleaved ? launch(r32, even) : launch(r32, halves);
  if (a.rot == 64) return a.interleaved ? launch(r64, even) : launch(r64, halves);
  if constexpr (D >= 128) {
    const std::integral_constant<int, 128> r128{};
    if (a.rot == 128) return a.interleaved ? launch(r128, even) : launch(r128, halves);
  }
  return hipErrorNotSupported;
}

}  // namespace kvattn
