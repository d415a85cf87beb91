// Writing new K and V rows into a cache in 8 bits: one workgroup's part, for the plain append
// and for the one that norms and rotates K first.
#pragma once

#include "common.hpp"
#include "kv_fp8.hpp"

namespace kvattn {

namespace {
constexpr int kBS = 16;
constexpr int kAppendWaves = 4;
constexpr int kWindow = 32;                     // tokens of a window
constexpr int kFewTokens = 512, kFewWindow = 2;    // up to kFewTokens tokens
constexpr int kSomeTokens = 2048, kSomeWindow = 8; // up to kSomeTokens
inline int append_window(int tokens) {
  return tokens <= kFewTokens ? kFewWindow : tokens <= kSomeTokens ? kSomeWindow : kWindow;
}
static_assert(kWindow + kBS <= kWave, "a window's slots and those its last run may reach");

typedef short s16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

// The byte of token r, dim j in a K or V tile.
__device__ __forceinline__ int k_place(int r, int j) { return (j / 16 * kBS + r) * 16 + j % 16; }
__device__ __forceinline__ int v_place(int r, int j) {
  return j / 64 * 1024 + r / 4 * 256 + j % 16 * 16 + j / 16 % 4 * 4 + r % 4;
}

constexpr uint32_t kInf = 0x7f800000u, kTop = 0x7f600000u;   // 448 * 2^119

// |x| as an integer that orders like it; 0 for what is not finite.
__device__ __forceinline__ uint32_t finite_bits(uint32_t x) {
  const uint32_t a = x & 0x7fffffffu;
  return a < kInf ? a : 0;
}

// The exponent byte of a largest value: |x| <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_byte(uint32_t amax) {
  return min(max((int)((amax + 0x1fffffu) >> 23) - 8, kFp8MinByte), kFp8MaxByte);
}

// x, or the largest value that has a code where it is finite and beyond that.
__device__ __forceinline__ uint32_t clamp_top(uint32_t x) {
  const uint32_t a = x & 0x7fffffffu;
  return a < kInf && a > kTop ? (x & 0x80000000u) | kTop : x;
}

// Four values of a 16-byte piece (which: 0, and 1 for a bf16 piece's second four)
// over the scale as four codes.
template <int ESZ>
__device__ __forceinline__ uint32_t encode4(uint4 x, int which, float scale) {
  s16x2_t r = {0, 0};
  if constexpr (ESZ == 2) {
    const uint32_t lo = which ? x.z : x.x, hi = which ? x.w : x.y;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, lo), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, hi), scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(x.x), __uint_as_float(x.y),
                                                 scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(x.z), __uint_as_float(x.w),
                                                 scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}

// Four codes times a power of two.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, r, true);
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t x) {
  const uint32_t y = __builtin_amdgcn_update_dpp(0, x, kCtrl, 0xf, 0xf, false);
  return x > y ? x : y;
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t x) {
  x = dpp_umax<kDppQuadSwap1>(x);
  x = dpp_umax<kDppQuadSwap2>(x);
  x = dpp_umax<kDppRowHalfMirror>(x);
  x = dpp_umax<kDppRowMirror>(x);
  const auto r16 = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = r16[0] > r16[1] ? r16[0] : r16[1];
  const auto r32 = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(r32[0] > r32[1] ? r32[0] : r32[1]);
}

// Dwords a and b of lane (16 s + c) are four dims of token s of a group of four;
// afterwards lanes below 32 have a's dims, those from 32 on b's, two of them each (2 (s % 2)
// and the next, in a and b), as dwords of the four tokens.
__device__ __forceinline__ void transpose_tokens(uint32_t& a, uint32_t& b) {
  const auto h = __builtin_amdgcn_permlane32_swap(a, b, false, false);   // tokens s % 2, s % 2 + 2
  uint32_t p = __builtin_amdgcn_perm(h[1], h[0], 0x05010400);   // dims 0, 1 of both
  uint32_t q = __builtin_amdgcn_perm(h[1], h[0], 0x07030602);   // dims 2, 3
  swap_rows16(p, q);                                            // p: tokens 0, 2; q: 1, 3
  a = __builtin_amdgcn_perm(q, p, 0x05010400);
  b = __builtin_amdgcn_perm(q, p, 0x07030602);
}
}  // namespace

// K rows as they come.
struct NoPrep {
  static constexpr bool kOn = false;
};

// The work of workgroup wg, of (windows x kv heads). ESZ: bytes per element of the new rows
// (2: bf16, 4: fp32), whose tokens lie k_stride and v_stride bytes apart. Prep: what
// is done to a K row, in fp32, before it is scaled.
template <int ESZ, int D, int kWin, class Prep>
__device__ __forceinline__ void append_fp8(
    int wg, const uint8_t* __restrict__ k_new, size_t k_stride, const uint8_t* __restrict__ v_new,
    size_t v_stride, const int* __restrict__ slot_mapping, uint8_t* __restrict__ kv,
    int num_tokens, int num_kv_heads, int capacity, const Prep& prep) {
  constexpr int kVec = 16 / ESZ;               // elements per load
  constexpr int kQ = kVec / 4;                 // dwords of codes per load
  constexpr int kCh = D / kVec;                // loads per row: 8, 16 or 32
  constexpr int kLoads = kBS * kCh / kWave;    // of a whole run
  constexpr int kTileBytes = kBS * D;
  constexpr int kParts = kTileBytes / (kWave * 16);   // 16-byte pieces per lane of a tile
  __shared__ __attribute__((aligned(16))) uint8_t stage[kAppendWaves][kTileBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x % kWave;
  const int g = wg % num_kv_heads;
  const int t0 = wg / num_kv_heads * kWin;

  // Slots of tokens t0 - 1 .. t0 + kWin + 14, one per lane; which tokens begin a run.
  const int t = t0 - 1 + lane;
  int slot = -1;
  if (lane < kWin + kBS && t >= 0 && t < num_tokens) slot = slot_mapping[t];
  const int block = (unsigned)slot < (unsigned)capacity ? slot / kBS : -1;
  const int before = __shfl_up(block, 1, kWave);
  const bool first = lane > 0 && lane <= kWin && block >= 0 && before != block;
  // the runs go on while tokens stay in one block, in order while slots follow each other
  const unsigned long long same = __ballot(lane > 0 && block >= 0 && before == block);
  const unsigned long long next = __ballot(lane > 0 && slot == __shfl_up(slot, 1, kWave) + 1);
  unsigned long long runs = __ballot(first);
  uint8_t* tile = stage[wave];

  // Token and 16-byte piece of a lane's i-th load: lanes 16 s .. 16 s + 15 have a token
  // s of every four.
  auto row_of = [&](int i) __attribute__((always_inline)) {
    const int s = lane / 16;
    return kCh == 8 ? 8 * i + lane % 16 / 8 * 4 + s : kCh == 16 ? 4 * i + s : i / 2 * 4 + s;
  };
  auto piece_of = [&](int i) __attribute__((always_inline)) {
    return kCh == 8 ? lane % 8 : kCh == 16 ? lane % 16 : i % 2 * 16 + lane % 16;
  };

  for (int task = 0; runs; ++task) {
    const int at = __builtin_ctzll(runs);        // lane of the run's first token
    if (task % 2) runs &= runs - 1;              // K, then V of each run
    if (task % kAppendWaves != wave) continue;
    const bool is_v = task % 2;
    const int n = min(kBS, 1 + (int)__builtin_ctzll(~(same >> (at + 1))));
    const int b = __builtin_amdgcn_readlane(block, at);
    const size_t stride = is_v ? v_stride : k_stride;
    const uint8_t* src =
        (is_v ? v_new : k_new) + (size_t)(t0 - 1 + at) * stride + (size_t)g * (D * ESZ);
    uint8_t* base = kv + (size_t)b * fp8_block_bytes(num_kv_heads, D);
    uint8_t* dst = base + (size_t)((is_v ? num_kv_heads : 0) + g) * kTileBytes;
    uint8_t* exp = base + fp8_tiles_bytes(num_kv_heads, D) + 2 * g + is_v;
    const int old = *exp;

    // ---- the run's rows, and their largest value ----
    uint4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      x[i] = make_uint4(0, 0, 0, 0);
      if (row_of(i) < n)
        x[i] = *reinterpret_cast<const uint4*>(src + (size_t)row_of(i) * stride + piece_of(i) * 16);
    }
    // a prepared row's values, which are in fp32 until they are codes
    const bool prepared = Prep::kOn && !is_v;
    float y[Prep::kOn ? kLoads * kVec : 1];
    uint32_t amax = 0;
    if (prepared) {
      if constexpr (Prep::kOn) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (ESZ == 2) {
              y[i * kVec + 2 * e] = bf16lo(u[e]);
              y[i * kVec + 2 * e + 1] = bf16hi(u[e]);
            } else {
              y[i * kVec + e] = __uint_as_float(u[e]);
            }
          }
        }
        constexpr int kPer = kCh > 16 ? kCh / 16 : 1;   // loads of a row
#pragma unroll
        for (int i = 0; i < kLoads; i += kPer)
          prep.apply(y + i * kVec, t0 - 1 + at + min(row_of(i), n - 1), piece_of(i));
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if (row_of(i) >= n) y[i * kVec + e] = 0.f;
            amax = max(amax, __float_as_uint(y[i * kVec + e]) & 0x7fffffffu);
          }
      }
    } else if constexpr (ESZ == 2) {
      u16x2_t m = {0, 0};
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          m = __builtin_elementwise_max(
              m, __builtin_bit_cast(u16x2_t, (&x[i].x)[e] & 0x7fff7fffu));
      amax = (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = max(amax, (&x[i].x)[e] & 0x7fffffffu);
    }
    amax = wave_umax(amax);
    if (amax >= kInf) {   // infinities and NaN do not count
      amax = 0;
      if (prepared) {
        if constexpr (Prep::kOn) {
#pragma unroll
          for (int e = 0; e < kLoads * kVec; ++e)
            amax = max(amax, finite_bits(__float_as_uint(y[e])));
        }
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w = (&x[i].x)[e];
            amax = max(amax, finite_bits(ESZ == 2 ? w & 0xffff0000u : w));
            if (ESZ == 2) amax = max(amax, finite_bits(w << 16));
          }
      }
      amax = wave_umax(amax);
    }
    if (amax > kTop) {    // values beyond the largest code at the largest exponent
      if constexpr (Prep::kOn) {
#pragma unroll
        for (int e = 0; e < kLoads * kVec; ++e)
          if (prepared) y[e] = __uint_as_float(clamp_top(__float_as_uint(y[e])));
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t& w = (&x[i].x)[e];
          w = ESZ == 2 ? clamp_top(w & 0xffff0000u) | clamp_top(w << 16) >> 16 : clamp_top(w);
        }
    }

    // ---- the block's exponent ----
    const unsigned long long mine = ((1ull << n) - 1) << at;
    const bool fresh = (__ballot(slot % kBS == 0) & mine) != 0;
    const int kept = min(max(old, kFp8MinByte), kFp8MaxByte);
    const int need = exponent_byte(amax);
    const int byte = __builtin_amdgcn_readfirstlane(fresh ? need : max(kept, need));
    const bool grown = !fresh && byte != kept;
    const bool ordered = n == kBS && ((next >> (at + 1)) & 0x7fff) == 0x7fff;
    // 16 powers of two add up to 2^16 - 1 only if they are all different ones
    const bool whole =
        ordered || (n == kBS && wave_sum(lane >= at && lane < at + n ? (float)(1 << (slot & 15))
                                                                     : 0.f) == 65535.f);
    if (lane == 0) *exp = (uint8_t)byte;

    // ---- the codes, in a tile in LDS ----
    if (grown && !whole) {
      const float by = fp8_scale(127 + max(kept - byte, -120));
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
        const uint4 w = *reinterpret_cast<const uint4*>(dst + (p * kWave + lane) * 16);
        *reinterpret_cast<uint4*>(tile + (p * kWave + lane) * 16) = make_uint4(
            rescale4(w.x, by), rescale4(w.y, by), rescale4(w.z, by), rescale4(w.w, by));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    const bool direct = !grown && !whole;
    uint8_t* to = direct ? dst : tile;
    const float scale = fp8_scale(byte);
    uint32_t w[kLoads * kQ];
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int c = 0; c < kQ; ++c) {
        if (prepared) {
          if constexpr (Prep::kOn) {
            const float* f = y + i * kVec + 4 * c;
            w[i * kQ + c] = encode4<4>(make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]),
                                                  __float_as_uint(f[2]), __float_as_uint(f[3])),
                                       0, scale);
          }
        } else {
          w[i * kQ + c] = encode4<ESZ>(x[i], c, scale);
        }
      }
    if (ordered && is_v) {
      // dwords of four tokens, the pairs (2 k, 2 k + 1) at a time
#pragma unroll
      for (int k = 0; k < kLoads * kQ; k += 2) {
        transpose_tokens(w[k], w[k + 1]);
        const int m = k + lane / 32, i = m / kQ;          // whose dims this lane has now
        const int r = row_of(0) / 4 * 4 + (kCh == 8 ? 8 * i : kCh == 16 ? 4 * i : i / 2 * 4);
        const int j = (kCh == 32 ? i % 2 * 16 + lane % 16 : piece_of(0)) * kVec + m % kQ * 4 +
                      lane / 16 % 2 * 2;
        *reinterpret_cast<uint32_t*>(tile + v_place(r, j)) = w[k];
        *reinterpret_cast<uint32_t*>(tile + v_place(r, j + 1)) = w[k + 1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = row_of(i);
        const int r = ordered ? row : __shfl(slot, at + min(row, n - 1), kWave) % kBS;
        if (row >= n) continue;
        const int j = piece_of(i) * kVec;
        if (!is_v) {
          if constexpr (kQ == 2)
            *reinterpret_cast<uint2*>(to + k_place(r, j)) = make_uint2(w[2 * i], w[2 * i + 1]);
          else
            *reinterpret_cast<uint32_t*>(to + k_place(r, j)) = w[i];
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            to[v_place(r, j + e)] = (uint8_t)(w[i * kQ + e / 4] >> (8 * (e % 4)));
        }
      }
    }
    if (direct) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int p = 0; p < kParts; ++p)
      *reinterpret_cast<uint4*>(dst + (p * kWave + lane) * 16) =
          *reinterpret_cast<const uint4*>(tile + (p * kWave + lane) * 16);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace kvattn
