// The 8-bit cache: where a block's tiles and exponents lie, and the walk of one
// wavefront over a run of a sequence's tokens in it.
//
// A tile is 16 tokens of one kv head's K or V in e4m3 with one power of two for all
// of it, kept as the exponent + 127 in a byte. A power of two loses nothing
// against a finer scale, since e4m3's relative step is the same in every binade;
// it makes code * 2^e exact in bf16 (4 significant bits, and the exponents in use keep
// it normal), so the products see the cache's values without a rounding; and a
// scale that is raised later moves the codes exactly but for those that
// leave the normal range. The bytes lie inside the block, so that one address per
// layer, block copies and the elastic range cover them as they do the tiles; a
// block is padded to 128 bytes, a cache line, so that tiles begin on one.
//
// The products run on the bf16 matrix instructions. The 8-bit ones (q split
// exactly into two e4m3 halves) would take the codes as they lie, but they align the
// products of a sum to its largest and drop what falls below: measured 2^-13
// of the sum of the terms' sizes, where the bf16 ones are at 2^-22 to 2^-26.
#pragma once

#include <type_traits>

#include "common.hpp"
#include "decode_walk.hpp"

namespace kvattn {

constexpr int kFp8MinByte = 10;    // 2^-117: the least code, 2^-9, stays normal in bf16
constexpr int kFp8MaxByte = 246;   // 2^119: 448 * 2^119 is finite in bf16

__host__ __device__ constexpr size_t fp8_tiles_bytes(int num_kv_heads, int head_dim) {
  return 2 * (size_t)num_kv_heads * 16 * head_dim;
}
__host__ __device__ constexpr size_t fp8_block_bytes(int num_kv_heads, int head_dim) {
  return fp8_tiles_bytes(num_kv_heads, head_dim) + ((2 * (size_t)num_kv_heads + 127) & ~size_t(127));
}

// Four codes (a dword) as bf16, times scale (a power of two): exact.
__device__ __forceinline__ uint2 fp8x4_to_bf16(uint32_t w, float scale) {
  const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
  const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
__device__ __forceinline__ bf16x8_t fp8x8_to_bf16(uint32_t a, uint32_t b, float sa, float sb) {
  const uint2 x = fp8x4_to_bf16(a, sa), y = fp8x4_to_bf16(b, sb);
  return __builtin_bit_cast(bf16x8_t, make_uint4(x.x, x.y, y.x, y.y));
}

__device__ __forceinline__ float fp8_scale(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// The bytes of the first n (clamped to 0 .. 4) of a dword.
__device__ __forceinline__ uint32_t first_bytes(int n) {
  return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
}

// Where a workgroup's tiles and exponents of one kv head lie.
struct Fp8Tiles {
  const uint8_t* kv;
  uint32_t block_bytes, k_off, v_off, e_off;   // at most 2^16 heads of 4 KiB
  __device__ __forceinline__ Fp8Tiles(const uint8_t* layer, int num_kv_heads, int head_dim, int g)
      : kv(layer),
        block_bytes((uint32_t)fp8_block_bytes(num_kv_heads, head_dim)),
        k_off((uint32_t)g * 16 * head_dim),
        v_off((uint32_t)(num_kv_heads + g) * 16 * head_dim),
        e_off((uint32_t)fp8_tiles_bytes(num_kv_heads, head_dim) + 2 * g) {}
  __device__ __forceinline__ const uint8_t* block(int id) const {
    return kv + (uint64_t)(uint32_t)id * block_bytes;
  }
};

// One wavefront's walk over tokens [t0, t1), as walk_bf16 with the cache in 8 bits.
// A load of 1 KiB is 64 dims of 16 tokens. Of K, lane l has 16 dims of token l % 16,
// two operands of eight once they are converted. Of V, the tile's order gives
// lane l tokens 4 (l / 16) .. + 4 of dims l % 16 + 16 w in dword w: with the
// same four tokens of a second block, the operand whose rows are 16 dims, and
// the tokens are those whose scores the lane has, so nothing is exchanged
// between lanes. The conversions (32 a block) take the place of the lane swaps
// that the bf16 walk needs there.
template <int D, int G, bool kAhead, class Score>
__device__ __forceinline__ void walk_fp8(const Fp8Tiles& tiles, const uint16_t* __restrict__ q,
                                         const int* __restrict__ bt, int num_blocks, int t0,
                                         int t1, const Score& how, float* o_out, float2* ml_out,
                                         int h0 = 0, int own = 0, int lo = 0) {
  const auto& score = how.held();
  constexpr int kBS = 16, kTile = 64, kTB = kTile / kBS;
  constexpr int kL = D / 64;   // loads per tile
  const int lane = threadIdx.x % kWave;
  const int head = lane % 16, row = lane / 16;
  // The exponents of the walk's next 64 blocks, one block per lane.
  auto walk_exps = [&](int id) __attribute__((always_inline)) {
    return id >= 0 ? (int)*reinterpret_cast<const uint16_t*>(tiles.block(id) + tiles.e_off) : 0;
  };
  int my_id = walk_ids(bt, t0, t1, num_blocks);
  int my_exp = walk_exps(my_id);
  bf16x8_t qreg[kL][2];
#pragma unroll
  for (int i = 0; i < kL; ++i)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      uint4 v = *reinterpret_cast<const uint4*>(q + min(head, G - 1) * D + i * 64 + row * 16 + b * 8);
      if (head >= G) v = make_uint4(0, 0, 0, 0);
      qreg[i][b] = __builtin_bit_cast(bf16x8_t, v);
    }

  float slope = 0.f;
  if constexpr (Score::kOn) slope = score.raw_slope(h0 + min(head, G - 1), q);
  float m_run = -INFINITY, l_run = 0.f;   // head's max; the lane's part of its sum
  f32x4_t acc[4 * kL];
#pragma unroll
  for (int i = 0; i < 4 * kL; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto load = [&](auto always, const int (&bid)[kTB], uint4 (&kreg)[kTB][kL],
                  uint4 (&vreg)[kTB][kL]) __attribute__((always_inline)) {
    constexpr bool kAlways = decltype(always)::value;
#pragma unroll
    for (int j = 0; j < kTB; ++j) {
      if (kAlways || bid[j] >= 0) {
        const uint8_t* bp = tiles.block(kAlways ? max(bid[j], 0) : bid[j]);
        const uint4* kp = reinterpret_cast<const uint4*>(bp + tiles.k_off) + lane;
        const uint4* vp = reinterpret_cast<const uint4*>(bp + tiles.v_off) + lane;
#pragma unroll
        for (int i = 0; i < kL; ++i) {
          kreg[j][i] = load_nt(kp + i * kWave);
          vreg[j][i] = load_nt(vp + i * kWave);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kL; ++i) {
          kreg[j][i] = make_uint4(0, 0, 0, 0);
          vreg[j][i] = make_uint4(0, 0, 0, 0);
        }
      }
    }
  };

  // Zeroes V's slots at or past t1, or before lo: they may hold anything, and zero times NaN
  // is NaN.
  auto cut = [&](int tb, uint4 (&vreg)[kTB][kL]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kTB; ++j) {
      const int tok = tb + j * kBS + row * 4;
      uint32_t keep = first_bytes(t1 - tok);
      if constexpr (Score::kOn) keep &= ~first_bytes(lo - tok);
#pragma unroll
      for (int i = 0; i < kL; ++i) {
        const uint4 v = vreg[j][i];
        vreg[j][i] = make_uint4(v.x & keep, v.y & keep, v.z & keep, v.w & keep);
      }
    }
  };
  // The products and softmax of one loaded step; tail: it may end inside a
  // block; zero: a block without a valid id still holds what was loaded for it.
  auto compute = [&](int tb, const int (&bid)[kTB], const int (&exps)[kTB], bool tail, bool zero,
                     const uint4 (&kreg)[kTB][kL],
                     uint4 (&vreg)[kTB][kL]) __attribute__((always_inline)) {
    // ---- scores ----
    float x[4 * kTB];
#pragma unroll
    for (int j = 0; j < kTB; ++j) {
      const float ks = fp8_scale(exps[j] & 0xff);
      f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kL; ++i) {
        const uint4 k = kreg[j][i];
        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8x8_to_bf16(k.x, k.y, ks, ks), qreg[i][0],
                                                     sc, 0, 0, 0);
        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8x8_to_bf16(k.z, k.w, ks, ks), qreg[i][1],
                                                     sc, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tok = tb + j * kBS + row * 4 + r;
        const bool keep = bid[j] >= 0 && (!tail || tok < t1);
        if constexpr (Score::kOn)
          x[4 * j + r] = sc[r];
        else
          x[4 * j + r] = keep ? sc[r] * score.scale_log2 : -INFINITY;
      }
    }
    if constexpr (Score::kOn) {
      score.template cap<false>(x);
      if (score.slopes) {
        const float by = slope * kLog2e, far = (float)(own - (tb + row * 4));
#pragma unroll
        for (int e = 0; e < 4 * kTB; ++e)
          x[e] = fmaf(by, (float)(e / 4 * kBS + e % 4) - far, x[e]);
      }
#pragma unroll
      for (int e = 0; e < 4 * kTB; ++e) {
        const int tok = tb + e / 4 * kBS + row * 4 + e % 4;
        x[e] = bid[e / 4] >= 0 && (!tail || tok < t1) && tok >= lo ? x[e] : -INFINITY;
      }
    }

    // ---- online softmax over the step (log2 domain) ----
    float mx = m_run;
#pragma unroll
    for (int j = 0; j < kTB; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[4 * j + r]);
    const float mn = cross_row_max(mx);
    const float ref = (mn == -INFINITY) ? 0.f : mn;
    const float alpha = fast_exp2(m_run - ref);
    m_run = mn;
    float psum = 0.f;
    uint2 pw[kTB];
#pragma unroll
    for (int j = 0; j < kTB; ++j) {
      pw[j].x = pack_bf16x2(fast_exp2(x[4 * j] - ref), fast_exp2(x[4 * j + 1] - ref));
      pw[j].y = pack_bf16x2(fast_exp2(x[4 * j + 2] - ref), fast_exp2(x[4 * j + 3] - ref));
      // A weight is rounded to bf16, as the matrix instruction takes it: at most 2^-8 of
      // it, the size of the output's own rounding, and independent from token to
      // token. The row sum adds the rounded weights, so that they still add up to one.
      psum = dot2_bf16(pw[j].x, kBf16OnePair, psum);
      psum = dot2_bf16(pw[j].y, kBf16OnePair, psum);
    }
    l_run = fmaf(l_run, alpha, psum);
#pragma unroll
    for (int i = 0; i < 4 * kL; ++i) acc[i] *= alpha;

    // ---- p . v, two blocks at a time ----
    if (zero && __builtin_expect((bid[0] | bid[1] | bid[2] | bid[3]) < 0, 0)) {
#pragma unroll
      for (int j = 0; j < kTB; ++j) {
        if (bid[j] >= 0) continue;
#pragma unroll
        for (int i = 0; i < kL; ++i) vreg[j][i] = make_uint4(0, 0, 0, 0);
      }
    }
    if (tail || (Score::kOn && !kAhead && tb < lo)) cut(tb, vreg);
#pragma unroll
    for (int j = 0; j < kTB; j += 2) {
      const float s0 = fp8_scale(exps[j] >> 8), s1 = fp8_scale(exps[j + 1] >> 8);
      const bf16x8_t b =
          __builtin_bit_cast(bf16x8_t, make_uint4(pw[j].x, pw[j].y, pw[j + 1].x, pw[j + 1].y));
#pragma unroll
      for (int i = 0; i < kL; ++i) {
        const uint4 v0 = vreg[j][i], v1 = vreg[j + 1][i];
        const uint32_t w0[4] = {v0.x, v0.y, v0.z, v0.w}, w1[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
        for (int w = 0; w < 4; ++w)
          acc[4 * i + w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              fp8x8_to_bf16(w0[w], w1[w], s0, s1), b, acc[4 * i + w], 0, 0, 0);
      }
    }
  };
  auto step_ids = [&](int tb, int (&bid)[kTB]) __attribute__((always_inline)) {
    const int at = (tb - t0) / kBS % kWave;
    if (!kAhead && at == 0 && tb != t0) {
      my_id = walk_ids(bt, tb, t1, num_blocks);
      my_exp = walk_exps(my_id);
    }
#pragma unroll
    for (int j = 0; j < kTB; ++j) bid[j] = __builtin_amdgcn_readlane(my_id, at + j);
  };
  // read where they are used, so that nothing waits for them before the step's loads
  auto step_exps = [&](int tb, int (&exps)[kTB]) __attribute__((always_inline)) {
    const int at = (tb - t0) / kBS % kWave;
#pragma unroll
    for (int j = 0; j < kTB; ++j) exps[j] = __builtin_amdgcn_readlane(my_exp, at + j);
  };

  constexpr std::true_type kAll{};
  constexpr std::false_type kReal{};
  if constexpr (!kAhead) {
    for (int tb = t0; tb < t1; tb += kTile) {
      int bid[kTB], exps[kTB];
      uint4 kreg[kTB][kL], vreg[kTB][kL];
      step_ids(tb, bid);
      load(kReal, bid, kreg, vreg);
      step_exps(tb, exps);
      compute(tb, bid, exps, tb + kTile > t1, false, kreg, vreg);
    }
  } else {
    int id_a[kTB], id_b[kTB], e_a[kTB], e_b[kTB];
    uint4 k_a[kTB][kL], v_a[kTB][kL], k_b[kTB][kL], v_b[kTB][kL];
    int tb = t0;
    step_ids(tb, id_a);
    load(kAll, id_a, k_a, v_a);
    if (Score::kOn && tb < lo) cut(tb, v_a);   // as in the bf16 walk
    for (;;) {
      if (tb + kTile >= t1) {
        step_exps(tb, e_a);
        compute(tb, id_a, e_a, tb + kTile > t1, true, k_a, v_a);
        break;
      }
      step_ids(tb + kTile, id_b);
      load(kAll, id_b, k_b, v_b);
      __builtin_amdgcn_sched_barrier(0);   // all of them before the step's products
      step_exps(tb, e_a);
      compute(tb, id_a, e_a, false, true, k_a, v_a);
      tb += kTile;
      if (tb + kTile >= t1) {
        step_exps(tb, e_b);
        compute(tb, id_b, e_b, tb + kTile > t1, true, k_b, v_b);
        break;
      }
      step_ids(tb + kTile, id_a);
      load(kAll, id_a, k_a, v_a);
      __builtin_amdgcn_sched_barrier(0);
      step_exps(tb, e_b);
      compute(tb, id_b, e_b, false, true, k_b, v_b);
      tb += kTile;
    }
  }

  const float l_tot = cross_row_sum(l_run);
  if (head < G) {
#pragma unroll
    for (int i = 0; i < 4 * kL; ++i)
      *reinterpret_cast<f32x4_t*>(o_out + head * D + i * 16 + row * 4) = acc[i];
    if (row == 0) ml_out[head] = make_float2(m_run, l_tot);
  }
}

}  // namespace kvattn
