// How a score is made of q . k: plainly scaled, or capped by a tanh, biased by distance and
// cut to a window.
#pragma once

#include "common.hpp"
#include "launch.hpp"

namespace kvattn {

constexpr int kNoWindow = 0x3fffffff;

// scale * q . k, causal.
struct PlainScore {
  static constexpr bool kOn = false;
  static constexpr int window = kNoWindow;
  float scale_log2;
  __device__ __forceinline__ const PlainScore& held() const { return *this; }
};

// a = scale q.k; a = cap tanh(a / cap); a += slope (key - row); keys from row - window + 1 on.
// All in the log2 domain.
enum class Cap { kNo, kYes, kAsk };   // known where the kernel is built, or asked for each score
template <Cap kCap>
struct ModScore {
  static constexpr bool kOn = true;
  float scale_log2;       // of q . k
  float cap_log2;         // 0: no cap
  float tanh_scale;       // a / cap of a q . k
  const float* slopes;    // of every query head, null: no bias
  int window;             // kNoWindow: none

  __device__ __forceinline__ bool has_cap() const {
    return kCap == Cap::kYes || (kCap == Cap::kAsk && cap_log2 > 0.f);
  }
  __device__ __forceinline__ float slope(int head) const {
    return slopes ? slopes[head] * kLog2e : 0.f;
  }
  // First key that the row at position pos sees.
  __device__ __forceinline__ int first_key(int pos) const { return max(0, pos - window + 1); }

  // cap tanh(dot scale / cap). Near zero by the odd polynomial that is nearest to tanh in
  // [0, 0.6], off by 8e-8 of it; from there on 1 - 2 / (e^2x + 1), whose error, 2^-22 of the
  // cap, is then small beside the value. kExact: the library's tanh, for fp32.
  template <bool kExact>
  __device__ __forceinline__ float capped(float dot) const {
    const float z = dot * tanh_scale;
    if constexpr (kExact) return cap_log2 * tanhf(z);
    const float w = z * z;
    float h = fmaf(w, kTanh[3], kTanh[2]);
    h = fmaf(h, w, kTanh[1]);
    h = fmaf(h, w, kTanh[0]);
    const float near = dot * scale_log2 * fmaf(h, w, 1.f);
    const float u = fast_exp2(z * (2.f * kLog2e));
    const float far = fmaf(-2.f * cap_log2, __builtin_amdgcn_rcpf(u + 1.f), cap_log2);
    return fabsf(z) < 0.6f ? near : far;
  }
  static constexpr float kTanh[4] = {-0.333326216f, 0.133135208f, -0.0522311078f, 0.0156404821f};

  // The same in vector registers: a walk's scalar ones are full of addresses.
  __device__ __forceinline__ ModScore held() const {
    ModScore s = *this;
    asm("" : "+v"(s.scale_log2), "+v"(s.cap_log2), "+v"(s.tanh_scale));
    return s;
  }

  // What a prefill tile does to its scores before its softmax (apply): nothing, and then
  // they only miss their scale, which is above zero so that masked ones may be minus
  // infinity; or all that makes them, for heads with a slope and without.
  enum Work : int { kNothing, kScale, kBias };
  __device__ __forceinline__ int work(float slope_log2) const {
    return slope_log2 != 0.f ? kBias : kCap == Cap::kYes || !(scale_log2 > 0.f) ? kScale : kNothing;
  }
  // Finishes the scores of 64 keys and 32 rows as a prefill tile's lane holds them: element e
  // of s[t] is key 32 t + 16 (e / 8) + 8 (lane / 32) + e % 8 of the step, whose first key is
  // rel tokens after the wavefront's first row; the row is lane % 32.
  template <typename V>
  __device__ __forceinline__ void apply(int work, V (&s)[2], int rel, float slope_log2,
                                        int lane) const {
    asm volatile("" : "+s"(work));   // compared here each time, not kept as masks over the loop
    if (kCap == Cap::kYes) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = capped<false>(s[t][e]);
    } else if (work != kNothing) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] *= scale_log2;
    }
    if (work == kBias) {
      const float b = slope_log2 * (float)(rel + lane / 32 * 8 - lane % 32);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[t][e] += fmaf(slope_log2, (float)(32 * t + e / 8 * 16 + e % 8), b);
    }
  }

  // The score of a key that lies ago tokens before the row.
  template <bool kExact>
  __device__ __forceinline__ float at(float dot, float slope_log2, int ago) const {
    const float x = has_cap() ? capped<kExact>(dot) : dot * scale_log2;
    return fmaf(slope_log2, -(float)ago, x);
  }
};

inline int window_keys(const ScoreMods& m) {
  return m.window > 0 && m.window < kNoWindow ? m.window : kNoWindow;
}

template <Cap kCap>
ModScore<kCap> mod_score(float scale, const ScoreMods& m) {
  ModScore<kCap> s;
  s.scale_log2 = scale * kLog2e;
  s.cap_log2 = m.softcap * kLog2e;
  s.tanh_scale = m.softcap > 0.f ? scale / m.softcap : 0.f;
  s.slopes = m.slopes;
  s.window = window_keys(m);
  return s;
}

}  // namespace kvattn
