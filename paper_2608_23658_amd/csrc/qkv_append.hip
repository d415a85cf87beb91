// What lies between a layer's projection and its attention, in one launch: norms of the q
// and k heads, their rotation by position, and the new K and V written into their paged
// slots (the paper, Section 3, "The contiguity constraint": one tensor per layer indexed by
// block id; Section 2: blocks of fixed size).
//
// The first workgroups have K and V, a wavefront one head's K or V of a run of tokens; the
// others have q. A wavefront has some heads of a run of 16 tokens one after another, the next
// one's rows on their way while one's are computed, so that the cosines and sines are read
// once and no wavefront waits for each of its loads in turn. Every row is read once and written
// once; about 10 operations a value leave HBM as the bound. Rows are read along the lanes, 128
// bytes or more of each at a time, and K and V turned through LDS into the tiles' order.
// 8192 tokens in order, 128 dims, bf16, inputs not in a cache; copying as many bytes takes 42 us:
//   a head's rows in the tile's order in registers, one head a wavefront,
//     V's dims stored one by one                                                   77.0 us
//   q along the lanes with loads ahead, K and V by blocks, V through LDS           57.2
//   K along the lanes and heads one after another with loads ahead too             51.5
//   both dims of a pair in a lane (LaneRows::kPairsIn)                             43.5
//   no private memory, addresses made where they are used (kv_rows)                39.9
// (32 query heads over 8; 16 over 16 83.4 -> 38.9). 256 scattered tokens: 14.5 us, of inputs not
// in a cache. There each of V's 2-byte elements goes into a 32-byte run of its own, a quarter of
// a million of them.
//
// A run of K or V is the tokens of one block where tokens follow each other in slot order, so
// that a block is written whole by one wavefront wherever a chunk begins in it; tokens
// that stand alone are taken by sixteens. Which run a token belongs to follows from its own
// slot and its neighbours': of a token whose neighbour has the next or the last slot, the run
// in which its block would begin; else its place in the list.

#include "common.hpp"
#include "launch.hpp"
#include "qkv_rows.hpp"

namespace kvattn {

// Heads h0 .. h1 of run k: K heads, then V heads.
template <int ESZ, int D, int kRotDim, bool kEven>
__device__ __forceinline__ void kv_rows(const QkvArgs& a, int k, int h0, int h1,
                                        uint4* stage) {
  using R = LaneRows<ESZ, D, kRotDim, kEven, true>;
  constexpr int kRows = kRunTokens * R::kLanes / kWave;   // rows of a lane
  constexpr int kN = kRows * R::kPer;                     // its 16-byte pieces
  const int lane = threadIdx.x % kWave;
  const int hkv = a.num_kv_heads;
  constexpr size_t kTile = (size_t)kRunTokens * D * ESZ;
  // Values before one is chosen: a choice among a's members became one of their addresses, which
  // kept a in private memory, 40 bytes a lane that every wavefront wrote and read back.
  const uint8_t *k_rows = a.k, *v_rows = a.v;
  const size_t k_stride = a.k_stride, v_stride = a.v_stride;

  // Lane l looks at token 16 (k - 1) + l; the run's are among lanes 1 .. 31.
  const int t = kRunTokens * (k - 1) + lane;
  int slot = -1;
  if (lane <= 2 * kRunTokens && t >= 0 && t < a.num_tokens) slot = a.slot_mapping[t];
  const bool real = (unsigned)slot < (unsigned)(a.num_blocks * kRunTokens);
  const int at = slot % kRunTokens;
  const bool follows = at > 0 && __shfl_up(slot, 1, kWave) == slot - 1 && lane > 0;
  const bool leads = at < kRunTokens - 1 && __shfl_down(slot, 1, kWave) == slot + 1 &&
                     lane < 2 * kRunTokens;
  const int first = follows || leads ? t - at + kRunTokens - 1 : t;
  const bool mine = real && lane > 0 && lane < 2 * kRunTokens && first >= kRunTokens * k &&
                    first < kRunTokens * (k + 1);
  const unsigned long long run = __ballot(mine);
  const int n = __popcll(run);
  if (n == 0) return;
  // the run's tokens, one per lane
  const int rank = __popcll(run & ((1ull << lane) - 1));
  const int packed = __builtin_amdgcn_ds_permute((mine ? rank : kWave - 1) * 4, lane);

  const int piece = lane % R::kLanes;
  const bool any_k = h0 < hkv;
  float w[R::kElems];
  if (any_k && a.k_weight) R::weights(a.k_weight, piece, w);
  for (int from = 0; from < n; from += kRunTokens) {   // 16 at a time, once where in order
    int tok[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int i16 = min(from + lane / R::kLanes + r * (kWave / R::kLanes), n - 1);
      tok[r] = kRunTokens * (k - 1) + __shfl(packed, i16, kWave);
    }
    auto load = [&](int h, uint4 (&x)[kN]) __attribute__((always_inline)) {
      const bool is_k = h < hkv;
      const uint8_t* src = (is_k ? k_rows : v_rows) + (size_t)(is_k ? h : h - hkv) * (D * ESZ);
      const size_t stride = is_k ? k_stride : v_stride;
      // addresses are made here: kept over the heads, one for each stride, they took the third
      // wavefront of a SIMD (178 registers instead of 168)
      int at = piece;
      asm volatile("" : "+v"(at));
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        int t = tok[r];
        asm volatile("" : "+v"(t));
#pragma unroll
        for (int p = 0; p < R::kPer; ++p)
          x[r * R::kPer + p] = load_nt(reinterpret_cast<const uint4*>(src + (size_t)t * stride) +
                                       at + R::kLanes * p);
      }
    };
    uint4 ahead[kN];
    load(h0, ahead);
    float c[kRows][R::kPairs], s[kRows][R::kPairs];
    if (any_k) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) R::turns(a, tok[r], piece, c[r], s[r]);
    }
    const int i16 = from + lane % 16;
    const bool live = i16 < n;
    const int my_slot = __shfl(slot, __shfl(packed, live ? i16 : from, kWave), kWave);
    const int s0 = __builtin_amdgcn_readfirstlane(my_slot);
    const bool whole =
        n - from >= kRunTokens && s0 % kRunTokens == 0 && __all(my_slot == s0 + lane % 16);
    uint8_t* block = a.kv + (size_t)(my_slot / kRunTokens) * (2 * (size_t)hkv * kTile);
    const int in_block = my_slot % kRunTokens;

    for (int h = h0; h < h1; ++h) {
      const bool is_v = h >= hkv;
      uint8_t* tile = block + (size_t)h * kTile;
      uint4 raw[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) raw[i] = ahead[i];
      if (h + 1 < h1) load(h + 1, ahead);
      if (!is_v) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          float x[R::kElems];
#pragma unroll
          for (int p = 0; p < R::kPer; ++p) R::P::widen(raw[r * R::kPer + p], x + p * R::kVec);
          if (a.k_weight) R::norm(x, w, a.eps);
          R::rotate(x, piece, c[r], s[r]);
#pragma unroll
          for (int p = 0; p < R::kPer; ++p) raw[r * R::kPer + p] = R::P::narrow(x + p * R::kVec);
        }
      }
      // Through LDS (rows padded against conflicts) from rows along the lanes to the tile's order.
      constexpr int kRowU4 = D * ESZ / 16 + 1, kVec = R::kVec, kParts = kRunTokens / kVec;
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int p = 0; p < R::kPer; ++p)
          stage[(lane / R::kLanes + r * (kWave / R::kLanes)) * kRowU4 + piece + R::kLanes * p] =
              raw[r * R::kPer + p];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (is_v && whole) {   // a dim's 16 slots leave as 16-byte pieces
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const int idx = i * kWave + lane, j = idx / kParts, part = idx % kParts;
          uint32_t v[4];
          if constexpr (ESZ == 2) {
            const uint16_t* in = reinterpret_cast<const uint16_t*>(stage) + j;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = in[(part * 8 + 2 * e) * kRowU4 * 8] |
                     (uint32_t)in[(part * 8 + 2 * e + 1) * kRowU4 * 8] << 16;
          } else {
            const uint32_t* in = reinterpret_cast<const uint32_t*>(stage) + j;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = in[(part * 4 + e) * kRowU4 * 4];
          }
          reinterpret_cast<uint4*>(tile)[idx] = make_uint4(v[0], v[1], v[2], v[3]);
        }
      } else if (live) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const int chunk = 4 * i + lane / 16;
          const uint4 x = stage[lane % 16 * kRowU4 + chunk];
          if (!is_v) {
            reinterpret_cast<uint4*>(tile)[chunk * kRunTokens + in_block] = x;
          } else {
            const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const int at = (chunk * kVec + e) * kRunTokens + in_block;
              if constexpr (ESZ == 2)
                reinterpret_cast<uint16_t*>(tile)[at] = (uint16_t)(u[e / 2] >> (16 * (e % 2)));
              else
                reinterpret_cast<uint32_t*>(tile)[at] = u[e];
            }
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <int ESZ, int D, int kRotDim, bool kEven>
__global__ __launch_bounds__(kQkvWaves * kWave) void qkv_append_kernel(QkvArgs a, int kv_wgs,
                                                                       QkvSplit kv, QkvSplit q) {
  __shared__ uint4 stage[kQkvWaves][kRunTokens * (D * ESZ / 16 + 1)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if ((int)blockIdx.x < kv_wgs) {
    const int h0 = (blockIdx.x % kv.groups * kQkvWaves + wave) * kv.per_wave;
    const int h1 = min(2 * a.num_kv_heads, h0 + kv.per_wave);
    if (h0 < h1) kv_rows<ESZ, D, kRotDim, kEven>(a, blockIdx.x / kv.groups, h0, h1, stage[wave]);
  } else {
    q_rows<ESZ, D, kRotDim, kEven>(a, blockIdx.x - kv_wgs, q.groups, q.per_wave);
  }
}

template <int ESZ, int D, int kRotDim, bool kEven>
static hipError_t launch_qkv_t(const QkvArgs& a) {
  const int runs = (int)(((long long)a.num_tokens + kRunTokens - 1) / kRunTokens);
  const QkvSplit q = qkv_split(runs, a.num_q_heads);
  // a token's run may be the one after that of its place in the list
  const QkvSplit kv = qkv_split(runs + 1, 2 * a.num_kv_heads);
  if (kv.workgroups + q.workgroups > 0x7fffffffLL / kQkvWaves) return hipErrorInvalidValue;
  trace_before(a.stream, "qkv_append");
  hipLaunchKernelGGL((qkv_append_kernel<ESZ, D, kRotDim, kEven>),
                     dim3((unsigned)(kv.workgroups + q.workgroups)), dim3(kQkvWaves * kWave), 0,
                     a.stream, a, (int)kv.workgroups, kv, q);
  trace_after(a.stream);
  return hipGetLastError();
}

template <int ESZ, int D>
static hipError_t launch_qkv_d(const QkvArgs& a) {
  return with_rotation<ESZ, D>(a, [&](auto rot, auto even) {
    return launch_qkv_t<ESZ, D, decltype(rot)::value, decltype(even)::value>(a);
  });
}

hipError_t launch_qkv_append(const QkvArgs& a) {
  if (a.num_tokens == 0) return hipSuccess;
  if (a.head_dim == 128) return a.esz == 2 ? launch_qkv_d<2, 128>(a) : launch_qkv_d<4, 128>(a);
  if (a.head_dim == 64) return a.esz == 2 ? launch_qkv_d<2, 64>(a) : launch_qkv_d<4, 64>(a);
  return hipErrorNotSupported;
}

}  // namespace kvattn
