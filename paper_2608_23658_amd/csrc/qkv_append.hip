// What lies between a layer's projection and its attention, in one launch: norms of the q
// and k heads, their rotation by position, and the new K and V written into their paged
// slots (the paper, Section 3, "The contiguity constraint": one tensor per layer indexed by
// block id; Section 2: blocks of fixed size).
//
// The first workgroups have K and V, a wavefront one head's K or V of a run of tokens; the
// others have q, some heads of a run of 16 tokens one after another, so that the cosines and
// sines are read once. Every row is read once and written once.
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

// One K (g < num_kv_heads) or V head of run k.
template <int ESZ, int D, int kRotDim, bool kEven>
__device__ __forceinline__ void kv_rows(const QkvArgs& a, int k, int g, uint4* stage) {
  using R = TileRows<ESZ, D, kRotDim * ESZ / 64, kEven>;
  const int lane = threadIdx.x % kWave;
  const int row = lane / 16;
  const int hkv = a.num_kv_heads;
  const bool is_v = g >= hkv;
  if (is_v) g -= hkv;
  constexpr size_t kTile = (size_t)kRunTokens * D * ESZ;

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

  R rows;
  const uint8_t* weight = is_v ? nullptr : a.k_weight;
  const uint8_t* src = is_v ? a.v : a.k;
  const size_t stride = is_v ? a.v_stride : a.k_stride;
  for (int from = 0; from < n; from += kRunTokens) {   // 16 at a time, once where in order
    const int i16 = from + lane % 16;
    const bool live = i16 < n;
    const int l = __shfl(packed, live ? i16 : from, kWave);
    const int my_slot = __shfl(slot, l, kWave), tok = kRunTokens * (k - 1) + l;
    const int s0 = __builtin_amdgcn_readfirstlane(my_slot);
    const bool whole =
        n - from >= kRunTokens && s0 % kRunTokens == 0 && __all(my_slot == s0 + lane % 16);
    uint4 raw[R::kN];
#pragma unroll
    for (int i = 0; i < R::kN; ++i)
      raw[i] = load_nt(reinterpret_cast<const uint4*>(src + (size_t)tok * stride +
                                                      (size_t)g * (D * ESZ)) + 4 * i + row);
    uint8_t* tile = a.kv + (size_t)(my_slot / kRunTokens) * (2 * (size_t)hkv * kTile) +
                    (size_t)((is_v ? hkv : 0) + g) * kTile;
    const int in_block = my_slot % kRunTokens;
    if (!is_v) {
      if (weight) rows.load_weight(weight);
      rows.load(a, tok);
      float x[R::kElems];
#pragma unroll
      for (int i = 0; i < R::kN; ++i) R::P::widen(raw[i], x + i * R::kVec);
      if (weight) rows.norm(x, a.eps);
      rows.rotate(x);
      if (live) {
        uint4* to = reinterpret_cast<uint4*>(tile);
#pragma unroll
        for (int i = 0; i < R::kN; ++i)
          to[(4 * i + row) * kRunTokens + in_block] = R::P::narrow(x + i * R::kVec);
      }
    } else if (whole) {
      // Through LDS (rows padded against conflicts): a dim's 16 slots leave as 16-byte pieces.
      constexpr int kRowU4 = D * ESZ / 16 + 1, kVec = R::kVec, kParts = kRunTokens / kVec;
#pragma unroll
      for (int i = 0; i < R::kN; ++i) stage[lane % 16 * kRowU4 + 4 * i + row] = raw[i];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < R::kN; ++i) {
        const int idx = i * kWave + lane, j = idx / kParts, part = idx % kParts;
        uint32_t w[4];
        if constexpr (ESZ == 2) {
          const uint16_t* in = reinterpret_cast<const uint16_t*>(stage) + j;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = in[(part * 8 + 2 * e) * kRowU4 * 8] |
                   (uint32_t)in[(part * 8 + 2 * e + 1) * kRowU4 * 8] << 16;
        } else {
          const uint32_t* in = reinterpret_cast<const uint32_t*>(stage) + j;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = in[(part * 4 + e) * kRowU4 * 4];
        }
        reinterpret_cast<uint4*>(tile)[idx] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else if (live) {
#pragma unroll
      for (int i = 0; i < R::kN; ++i) {
        const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
        const int j0 = (4 * i + row) * R::kVec;
        if constexpr (ESZ == 2) {
          uint16_t* v = reinterpret_cast<uint16_t*>(tile);
#pragma unroll
          for (int e = 0; e < R::kVec; ++e)
            v[(j0 + e) * kRunTokens + in_block] = (uint16_t)(u[e / 2] >> (16 * (e % 2)));
        } else {
          uint32_t* v = reinterpret_cast<uint32_t*>(tile);
#pragma unroll
          for (int e = 0; e < R::kVec; ++e) v[(j0 + e) * kRunTokens + in_block] = u[e];
        }
      }
    }
  }
}

template <int ESZ, int D, int kRotDim, bool kEven>
__global__ __launch_bounds__(kQkvWaves * kWave) void qkv_append_kernel(QkvArgs a, int kv_wgs,
                                                                       int groups, int per_wave) {
  __shared__ uint4 stage[kQkvWaves][kRunTokens * (D * ESZ / 16 + 1)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if ((int)blockIdx.x < kv_wgs) {
    const int task = blockIdx.x * kQkvWaves + wave, heads = 2 * a.num_kv_heads;
    kv_rows<ESZ, D, kRotDim, kEven>(a, task / heads, task % heads, stage[wave]);
  } else {
    q_rows<ESZ, D, kRotDim, kEven>(a, blockIdx.x - kv_wgs, groups, per_wave);
  }
}

template <int ESZ, int D, int kRotDim, bool kEven>
static hipError_t launch_qkv_t(const QkvArgs& a) {
  // a token's run may be the one after that of its place in the list
  const long long runs = ((long long)a.num_tokens + kRunTokens - 1) / kRunTokens + 1;
  const long long kv_wgs = (runs * 2 * a.num_kv_heads + kQkvWaves - 1) / kQkvWaves;
  const QkvSplit s = qkv_split(a.num_tokens, a.num_q_heads);
  if (kv_wgs + s.workgroups > 0x7fffffffLL / kQkvWaves) return hipErrorInvalidValue;
  trace_before(a.stream, "qkv_append");
  hipLaunchKernelGGL((qkv_append_kernel<ESZ, D, kRotDim, kEven>),
                     dim3((unsigned)(kv_wgs + s.workgroups)), dim3(kQkvWaves * kWave), 0, a.stream,
                     a, (int)kv_wgs, s.groups, s.per_wave);
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
