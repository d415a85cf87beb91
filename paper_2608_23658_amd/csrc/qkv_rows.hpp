// Norm and rotation of q and k rows in registers.
#pragma once

#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace kvattn {

namespace {
constexpr int kRunTokens = 16;   // tokens of a run, slots of a block
constexpr int kQkvWaves = 4;
}  // namespace

// ESZ: bytes of an element. Values are fp32 between a row's load and its store.
template <int ESZ>
struct QkvPieces {
  static constexpr int kVec = 16 / ESZ;   // elements of a 16-byte piece
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
};

// (a, b) turned by an angle of cosine c and sine s.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float a1 = fmaf(a, c, -(b * s));
  b = fmaf(b, c, a * s);
  a = a1;
}

// The cosines and sines of n = 2 or 4 pairs from p on, at position pos. One outside the table
// gives NaN. p is a multiple of n, a table's row of 4 floats.
template <int kRotDim, int n>
__device__ __forceinline__ void load_turns_at(const QkvArgs& a, int pos, int p, float* c,
                                              float* s) {
  const bool in = (unsigned)pos < (unsigned)a.table_len;
  const float* at = a.table + (size_t)(in ? pos : 0) * kRotDim + p;
  if constexpr (n == 4) {
    const float4 x = *reinterpret_cast<const float4*>(at);
    const float4 y = *reinterpret_cast<const float4*>(at + kRotDim / 2);
    c[0] = x.x; c[1] = x.y; c[2] = x.z; c[3] = x.w;
    s[0] = y.x; s[1] = y.y; s[2] = y.z; s[3] = y.w;
  } else {
    const float2 x = *reinterpret_cast<const float2*>(at);
    const float2 y = *reinterpret_cast<const float2*>(at + kRotDim / 2);
    c[0] = x.x; c[1] = x.y;
    s[0] = y.x; s[1] = y.y;
  }
  if (!in) {
#pragma unroll
    for (int e = 0; e < n; ++e) c[e] = s[e] = NAN;
  }
}

// The cosines and sines of pairs p .. p + n of token t, n 2 or a multiple of 4 that p is a
// multiple of.
template <int kRotDim, int n>
__device__ __forceinline__ void load_turns(const QkvArgs& a, int t, int p, float* c, float* s) {
  constexpr int kHalf = kRotDim / 2, kStep = n % 4 == 0 ? 4 : 2;
  auto axis_of = [&](int pair) __attribute__((always_inline)) {
    return (pair >= a.axis_end[0]) + (pair >= a.axis_end[1]) + (pair >= a.axis_end[2]);
  };
  if (a.axis_end[0] >= kHalf) {   // one axis
    const int pos = a.positions[t];
#pragma unroll
    for (int e = 0; e < n; e += kStep) load_turns_at<kRotDim, kStep>(a, pos, p + e, c + e, s + e);
    return;
  }
#pragma unroll
  for (int e = 0; e < n; e += kStep) {
    const int axis = axis_of(p + e);
    if (axis == axis_of(p + e + kStep - 1)) {   // no section ends among them
      load_turns_at<kRotDim, kStep>(a, a.positions[(size_t)axis * a.num_tokens + t], p + e, c + e,
                                    s + e);
    } else {
#pragma unroll
      for (int i = e; i < e + kStep; ++i) {
        const int pos = a.positions[(size_t)axis_of(p + i) * a.num_tokens + t];
        const bool in = (unsigned)pos < (unsigned)a.table_len;
        const float* at = a.table + (size_t)(in ? pos : 0) * kRotDim + p + i;
        c[i] = in ? at[0] : NAN;
        s[i] = in ? at[kHalf] : NAN;
      }
    }
  }
}

// ---- rows along the lanes ----
// A row's 16-byte pieces lie in 8 or 16 neighbouring lanes (512 bytes: two in each of 16),
// so that rows are read and written as they lie. kRotDim 0: no rotation. kPairsIn: a row
// of 256 bytes whose pairs are its halves has two pieces in each of 8 lanes, so that a
// lane has both of a pair and a pair's cosine and sine are read once.
template <int ESZ, int D, int kRotDim, bool kEven, bool kPairsIn>
struct LaneRows {
  using P = QkvPieces<ESZ>;
  static constexpr int kVec = P::kVec, kCh = D / kVec;
  static constexpr bool kHalves = kPairsIn && !kEven && kRotDim == D && kCh == 16;
  static constexpr int kPer = kHalves || kCh > 16 ? 2 : 1;   // pieces of a row in a lane
  static constexpr int kLanes = kCh / kPer;                  // lanes of a row, pieces apart
  static constexpr int kElems = kPer * kVec;
  static constexpr int kOff = kRotDim / 2 / kVec;        // pieces between the two of a pair
  static constexpr bool kInLane = kEven || kOff == kLanes;   // both of a pair in a lane
  static constexpr int kPairs = kRotDim == 0 ? 1 : kInLane ? kElems / 2 : kVec;

  // The cosines and sines that a lane with pieces piece, piece + kLanes needs of token t.
  static __device__ __forceinline__ void turns(const QkvArgs& a, int t, int piece, float (&c)[kPairs],
                                               float (&s)[kPairs]) {
    if constexpr (kRotDim > 0) {
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        if constexpr (kEven) {
          if ((piece + kLanes * p) * kVec < kRotDim)
            load_turns<kRotDim, kVec / 2>(a, t, (piece + kLanes * p) * (kVec / 2), c + p * (kVec / 2),
                                          s + p * (kVec / 2));
        } else if constexpr (kInLane) {
          if (p < kPer / 2)
            load_turns<kRotDim, kVec>(a, t, (piece + kLanes * p) * kVec, c + p * kVec, s + p * kVec);
        } else if (p == 0 && piece < 2 * kOff) {
          load_turns<kRotDim, kVec>(a, t, piece % kOff * kVec, c, s);
        }
      }
    }
  }
  static __device__ __forceinline__ void weights(const uint8_t* weight, int piece,
                                                 float (&w)[kElems]) {
#pragma unroll
    for (int p = 0; p < kPer; ++p)
      P::widen(reinterpret_cast<const uint4*>(weight)[piece + kLanes * p], w + p * kVec);
  }
  // x * rsqrt(mean(x^2) + eps) * w
  static __device__ __forceinline__ void norm(float* x, const float (&w)[kElems], float eps) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kElems; ++e) sum = fmaf(x[e], x[e], sum);
    sum += dpp_mov<kDppQuadSwap1>(sum);
    sum += dpp_mov<kDppQuadSwap2>(sum);
    sum += dpp_mov<kDppRowHalfMirror>(sum);
    if constexpr (kLanes > 8) sum += dpp_mov<kDppRowMirror>(sum);
    const float by = rsqrtf(fmaf(sum, 1.f / D, eps));
#pragma unroll
    for (int e = 0; e < kElems; ++e) x[e] = x[e] * by * w[e];
  }
  // The same dim of the piece kOff lanes away in the row (xor).
  static __device__ __forceinline__ float across(float x) {
    if constexpr (kOff == 8) return dpp_mov<0x128>(x);          // rotate 16 lanes by 8
    if constexpr (kOff == 2) return dpp_mov<kDppQuadSwap2>(x);
    if constexpr (kOff == 4) return dpp_mov<kDppRowHalfMirror>(dpp_mov<0x1b>(x));   // 7 - (3 - i)
    return x;
  }
  static __device__ __forceinline__ void rotate(float* x, int piece, const float (&c)[kPairs],
                                                const float (&s)[kPairs]) {
    if constexpr (kRotDim == 0) return;
    if constexpr (kEven) {
#pragma unroll
      for (int p = 0; p < kPer; ++p)
        if ((piece + kLanes * p) * kVec < kRotDim) {
#pragma unroll
          for (int m = 0; m < kVec / 2; ++m)
            turn(x[p * kVec + 2 * m], x[p * kVec + 2 * m + 1], c[p * (kVec / 2) + m],
                 s[p * (kVec / 2) + m]);
        }
    } else if constexpr (kInLane) {
#pragma unroll
      for (int e = 0; e < kElems / 2; ++e) turn(x[e], x[e + kElems / 2], c[e], s[e]);
    } else {
      const bool in = piece < 2 * kOff, second = piece & kOff;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float other = across(x[e]);
        const float y = fmaf(x[e], c[e], second ? other * s[e] : -other * s[e]);
        x[e] = in ? y : x[e];
      }
    }
  }
};

// The q rows of workgroup wg, of (runs x groups of heads): per_wave heads a wavefront, the
// next one's rows on their way while one's are computed.
template <int ESZ, int D, int kRotDim, bool kEven>
__device__ __forceinline__ void q_rows(const QkvArgs& a, int wg, int groups, int per_wave) {
  using R = LaneRows<ESZ, D, kRotDim, kEven, true>;
  constexpr int kRows = kRunTokens * R::kLanes / kWave;   // rows of a lane
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int hq = a.num_q_heads;
  const int h0 = (wg % groups * kQkvWaves + wave) * per_wave;
  const int h1 = min(hq, h0 + per_wave);
  if (h0 >= h1) return;
  const int t0 = wg / groups * kRunTokens + lane / R::kLanes, piece = lane % R::kLanes;
  auto token = [&](int r) { return t0 + r * (kWave / R::kLanes); };
  auto load = [&](int h, uint4 (&x)[kRows * R::kPer]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int p = 0; p < R::kPer; ++p)
        x[r * R::kPer + p] =
            load_nt(reinterpret_cast<const uint4*>(
                        a.q + (size_t)min(token(r), a.num_tokens - 1) * a.q_stride +
                        (size_t)h * (D * ESZ)) + piece + R::kLanes * p);
  };
  uint4 next[kRows * R::kPer];
  load(h0, next);
  float w[R::kElems];
  if (a.q_weight) R::weights(a.q_weight, piece, w);
  float c[kRows][R::kPairs], s[kRows][R::kPairs];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    R::turns(a, min(token(r), a.num_tokens - 1), piece, c[r], s[r]);
  for (int h = h0; h < h1; ++h) {
    uint4 raw[kRows * R::kPer];
#pragma unroll
    for (int i = 0; i < kRows * R::kPer; ++i) raw[i] = next[i];
    if (h + 1 < h1) load(h + 1, next);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      float x[R::kElems];
#pragma unroll
      for (int p = 0; p < R::kPer; ++p) R::P::widen(raw[r * R::kPer + p], x + p * R::kVec);
      if (a.q_weight) R::norm(x, w, a.eps);
      R::rotate(x, piece, c[r], s[r]);
      if (token(r) < a.num_tokens) {
        uint4* to = reinterpret_cast<uint4*>(a.q_out + ((size_t)token(r) * hq + h) * (D * ESZ));
#pragma unroll
        for (int p = 0; p < R::kPer; ++p) to[piece + R::kLanes * p] = R::P::narrow(x + p * R::kVec);
      }
    }
  }
}

// How rows are dealt to wavefronts: more heads to each where there are enough to fill the
// card anyway. 8192 / 2048 tokens, 32 query heads over 8: at these bounds 39.9 / 17.1 us, at half
// of them 39.9 / 16.4 (but 1777 tokens of 12 over 3 in fp32 9.6 instead of 9.3), at twice
// 38.8 / 19.1 (4096 tokens of 64 over 8, 8 bits, 42.2 instead of 39.5). Then as many to each of a
// workgroup's wavefronts (46 heads over 1: 46.2 -> 42.0 us).
struct QkvSplit {
  int per_wave, groups;   // heads of a wavefront, workgroups of a run
  long long workgroups;
};
inline QkvSplit qkv_split(long long runs, int heads) {
  QkvSplit s;
  s.per_wave = runs * heads > 8192 ? 8 : runs * heads > 4096 ? 4 : runs * heads > 2048 ? 2 : 1;
  s.groups = (heads + kQkvWaves * s.per_wave - 1) / (kQkvWaves * s.per_wave);
  s.per_wave = (heads + kQkvWaves * s.groups - 1) / (kQkvWaves * s.groups);   // in even parts
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
