// How a score is made of q . k: plainly scaled, or capped by a tanh, biased by distance and
// cut to a window.
#pragma once

#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "launch.hpp"
#include "window.hpp"

namespace kvattn {

// What the scores of a kernel can be; all but plain ones have a window. kAny asks for each
// score.
enum class Form { kPlain, kWindow, kBias, kCap, kAny };

// scale * q . k, causal.
struct PlainScore {
  static constexpr bool kOn = false;
  static constexpr Form form = Form::kPlain;
  static constexpr int window = kNoWindow;
  float scale_log2;
  __device__ __forceinline__ const PlainScore& held() const { return *this; }
};

// The odd polynomial nearest to tanh in [0, 0.5] (off by 7e-7 of it): z + z^3 (c0 + c1 z^2 + ..).
constexpr float kTanh3[3] = {-0.333282646f, 0.132067148f, -0.0447894702f};
// kTanh3 in y = 2 log2(e) z.
constexpr float kTanhY[3] = {-0.0400316641f, 0.00190535828f, -7.76155430e-05f};

// a = scale q.k; a = cap tanh(a / cap); a += slope (key - row); keys from row - window + 1 on.
// All in the log2 domain.
template <Form kForm>
struct ModScore {
  static constexpr bool kOn = true;
  static constexpr Form form = kForm;
  float scale_log2;       // of q . k
  float cap_log2;         // 0: no cap
  float tanh_scale;       // a / cap of a q . k
  float exp_scale;        // 2 log2(e) times that
  const float* slopes;    // of every query head, null: no bias
  int window;             // kNoWindow: none
  // With a cap, of products smaller than near: a score is dot (p0 + p1 dot^2 + p2 dot^4 +
  // p3 dot^6), by kTanh3.
  float near, p0, p1, p2, p3;

  __device__ __forceinline__ bool has_cap() const {
    return kForm == Form::kCap || (kForm == Form::kAny && cap_log2 > 0.f);
  }
  __device__ __forceinline__ float slope(int head) const {
    return slopes ? slopes[head] * kLog2e : 0.f;
  }
  // First key that the row at position pos sees.
  __device__ __forceinline__ int first_key(int pos) const {
    return kvattn::first_key(pos, window);
  }

  // cap tanh(dot scale / cap) as cap (1 - 2 / (e^2x + 1)), off by 2^-22 of the cap, which for
  // one up to kSmallCap is 2^-14 of a weight. kExact: the library's tanh.
  static constexpr float kSmallCap = 256.f;   // in the log2 domain
  static __device__ __forceinline__ float capped_far(float dot, float exp_scale, float cap_log2) {
    const float u = fast_exp2(dot * exp_scale);
    return fmaf(-2.f * cap_log2, __builtin_amdgcn_rcpf(u + 1.f), cap_log2);
  }
  // The one or the other by the product's size, where a cap is large: off by 2^-19 of the
  // score. In y = 2 log2(e) z, which the exponential takes, so that a prefill tile needs no
  // register more.
  static __device__ __forceinline__ float capped_each(float dot, float exp_scale, float cap_log2,
                                                      float scale_log2) {
    const float y = dot * exp_scale, w = y * y;
    const float h = fmaf(fmaf(w, kTanhY[2], kTanhY[1]), w, kTanhY[0]);
    const float far = capped_far(dot, exp_scale, cap_log2);
    return fabsf(y) < kLog2e ? dot * scale_log2 * fmaf(h, w, 1.f) : far;
  }

  // ---- for a walk, some scores at a time ----

  // The same in vector registers: a walk's scalar ones are full of addresses.
  __device__ __forceinline__ ModScore held() const {
    ModScore s = *this;
    asm("" : "+v"(s.scale_log2), "+v"(s.cap_log2), "+v"(s.exp_scale));
    return s;
  }
  // A head's slope, times log2(e) where it is used: a load that nothing waits for here, from
  // any address that can be read where there is no bias.
  __device__ __forceinline__ float raw_slope(int head, const void* any) const {
    return *(slopes ? slopes + head : reinterpret_cast<const float*>(any));
  }
  // The scores of n products in place. kExact: with the library's tanh.
  template <bool kExact, int n>
  __device__ __forceinline__ void cap(float (&x)[n]) const {
    // a wavefront's branches on it are scalar ones
    const float c = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(cap_log2)));
    if (!(kForm == Form::kCap || (kForm == Form::kAny && c > 0.f))) {
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] *= scale_log2;
    } else if constexpr (kExact) {
#pragma unroll
      for (int e = 0; e < n; ++e) {
        // where tanh z is z to fp32, without the quotient of scale and cap, which may underflow
        const float z = x[e] * tanh_scale, y = cap_log2 * tanhf(z);
        x[e] = fabsf(z) < 0x1p-12f ? x[e] * scale_log2 : y;
      }
    } else if (c <= kSmallCap) {
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] = capped_far(x[e], exp_scale, cap_log2);
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] = capped_each(x[e], exp_scale, cap_log2, scale_log2);
    }
  }

  // ---- for a prefill tile, the scores of 64 keys and 32 rows at a time ----
  // As a lane holds them: element e is key key_of(e) + 8 (lane / 32) of the step, whose first
  // key is rel tokens after the wavefront's first row; the row is lane % 32.

  static __device__ __forceinline__ constexpr int key_of(int e) {
    return e / 16 * 32 + e / 8 % 2 * 16 + e % 8;
  }
  // How the softmax finds a step's scores, with its reference r taken off.
  struct Step {
    float by;               // times this
    float slope, ago;       // kBias: the bias of element e is slope (key_of(e) + ago)
    __device__ __forceinline__ float at(float dot, int e, float r) const {
      if constexpr (kForm == Form::kBias)
        return fmaf(dot, by, fmaf(slope, (float)key_of(e), fmaf(slope, ago, -r)));
      return fmaf(dot, by, -r);
    }
  };

  // Values in vector registers from here on: not hoisted out of a tile's loop, which has none
  // to spare.
  static __device__ __forceinline__ void hold(float& x) { asm volatile("" : "+v"(x)); }
  template <typename... T>
  static __device__ __forceinline__ void here(T&... x) {
    (hold(x), ...);
  }
  // Prepares a step's scores s, before they are masked: capped ones, and those of a scale that
  // is not above zero, are finished; others the softmax finishes beside the matrix work.
  template <typename V>
  __device__ __forceinline__ Step prepare(V (&s)[2], int rel, const float& slope_log2,
                                          int lane) const {
    const float at_lane = (float)(rel + lane / 32 * 8 - lane % 32);
    if constexpr (kForm == Form::kCap) {
      if (all_near(s)) {
        float c0 = p0, c1 = p1, c2 = p2, c3 = p3;
        here(c0, c1, c2, c3);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const float x = s[e / 16][e % 16], t = x * x;
          s[e / 16][e % 16] = x * fmaf(fmaf(fmaf(t, c3, c2), t, c1), t, c0);
        }
      } else if (small_cap()) {
        float scale = exp_scale, cap = cap_log2;
        here(scale, cap);
#pragma unroll
        for (int e = 0; e < 32; ++e)
          s[e / 16][e % 16] = capped_far(s[e / 16][e % 16], scale, cap);
      } else {
        // each by its own size: one large product must not cost the others' scores
        float scale = exp_scale, cap = cap_log2, near = p0;
        here(scale, cap, near);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          s[e / 16][e % 16] = capped_each(s[e / 16][e % 16], scale, cap, near);
          __builtin_amdgcn_sched_barrier(0);   // no registers for more at a time
        }
      }
      const float slope =
          __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(slope_log2)));
      if (slope != 0.f) {
        float at = at_lane, by = slope;
        here(at, by);
        const float first = by * at;
#pragma unroll
        for (int e = 0; e < 32; ++e)
          s[e / 16][e % 16] += fmaf(by, (float)key_of(e), first);
      }
      return {1.f, 0.f, 0.f};
    } else {
      if (scale_log2 > 0.f) return {scale_log2, slope_log2, at_lane};
      // masked scores are minus infinity before a scale above zero
#pragma unroll
      for (int e = 0; e < 32; ++e) s[e / 16][e % 16] *= scale_log2;
      return {1.f, slope_log2, at_lane};
    }
  }
  // cap_log2 <= kSmallCap, compared by its bits each time: no mask is kept.
  __device__ __forceinline__ bool small_cap() const {
    uint32_t c = __float_as_uint(cap_log2);
    asm volatile("" : "+s"(c));
    return c <= __float_as_uint(kSmallCap);
  }
  // Whether all of a wavefront's products are smaller than near.
  template <typename V>
  __device__ __forceinline__ bool all_near(const V (&s)[2]) const {
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      float r;
      asm("v_max3_f32 %0, |%1|, |%2|, %3"
          : "=v"(r) : "v"(s[e / 16][e % 16]), "v"(s[e / 16][e % 16 + 1]), "v"(m));
      m = r;
    }
    return __builtin_amdgcn_ballot_w64(!(m < near)) == 0;
  }
};

inline int window_keys(const ScoreMods& m) {
  return m.window > 0 && m.window < kNoWindow ? m.window : kNoWindow;
}

template <Form kForm>
ModScore<kForm> mod_score(float scale, const ScoreMods& m) {
  ModScore<kForm> s;
  s.scale_log2 = scale * kLog2e;
  s.cap_log2 = m.softcap * kLog2e;
  s.tanh_scale = m.softcap > 0.f ? scale / m.softcap : 0.f;
  s.exp_scale = s.tanh_scale * (2.f * kLog2e);
  s.slopes = m.slopes;
  s.window = window_keys(m);
  const float w = s.tanh_scale * s.tanh_scale;
  s.p0 = s.scale_log2;
  s.p1 = s.p0 * w * kTanh3[0];
  s.p2 = s.p0 * w * w * kTanh3[1];
  s.p3 = s.p0 * w * w * w * kTanh3[2];
  // A coefficient below fp32's normal range (a tiny scale, a large cap) is left out, and what is
  // near ends where its term would be 2^-22 of the score.
  float z = 0.5f;
  if (!std::isnormal(s.p3)) z = 0.13f;
  if (!std::isnormal(s.p2)) z = 0.036f;
  if (!std::isnormal(s.p1)) z = 8e-4f;
  // past the range none is near (a tiny cap), nor are products whose squares are
  s.near = w < 1e9f && std::isfinite(s.p3) ? std::min(z / std::fabs(s.tanh_scale), 1.8e19f) : 0.f;
  if (z < 0.5f) s.p3 = 0.f;
  if (z < 0.13f) s.p2 = 0.f;
  if (z < 0.036f) s.p1 = 0.f;
  return s;
}

// Calls launch with a call's scores in their form's type.
template <typename Launch>
hipError_t with_form(float scale, const ScoreMods& m, Launch launch) {
  if (m.softcap > 0.f) return launch(mod_score<Form::kCap>(scale, m));
  if (m.slopes) return launch(mod_score<Form::kBias>(scale, m));
  return launch(mod_score<Form::kWindow>(scale, m));
}

}  // namespace kvattn
