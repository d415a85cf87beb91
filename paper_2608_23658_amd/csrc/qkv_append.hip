// What lies between a layer's projection and its attention, in one launch: norms of the q
// and k heads, their rotation by position, and the new K and V written into their paged
// slots (the paper, Section 3, "The contiguity constraint": one tensor per layer indexed by
// block id; Section 2: blocks of fixed size).
//
// A wavefront takes a run of 16 consecutive tokens and some of the heads (q, k and v
// alike), one head after another, so that the cosines and sines of its tokens are read
// once. Every row is read once and written once.

#include "common.hpp"
#include "launch.hpp"
#include "qkv_rows.hpp"

namespace kvattn {

namespace {
constexpr int kBS = 16;        // slots per block, tokens per run
constexpr int kQkvWaves = 4;
}  // namespace

template <int ESZ, int D, int kRot, bool kEven>
__global__ __launch_bounds__(kQkvWaves * kWave) void qkv_append_kernel(QkvArgs a, int groups,
                                                                       int per_wave) {
  using R = QkvRows<ESZ, D, kRot, kEven>;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int row = lane / 16;
  const int hq = a.num_q_heads, hkv = a.num_kv_heads, heads = hq + 2 * hkv;
  const int h0 = (int)(blockIdx.x % groups * kQkvWaves + wave) * per_wave;
  const int h1 = min(heads, h0 + per_wave);
  if (h0 >= h1) return;
  const int t = (int)(blockIdx.x / groups) * kBS + lane % 16;
  const bool real = t < a.num_tokens;
  const int tc = min(t, a.num_tokens - 1);

  R rows;
  if (h0 < hq + hkv) rows.load_turns(a, tc);
  uint8_t* block = nullptr;    // of the token's slot; null: it has none
  int slot = 0;
  constexpr size_t kTile = (size_t)kBS * D * ESZ;
  if (h1 > hq && real) {
    slot = a.slot_mapping[t];
    if ((unsigned)slot < (unsigned)(a.num_blocks * kBS)) {
      block = a.kv + (size_t)(slot / kBS) * (2 * (size_t)hkv * kTile);
      slot %= kBS;
    }
  }

  const uint8_t* weight = nullptr;
  for (int h = h0; h < h1; ++h) {
    const bool is_q = h < hq, is_v = h >= hq + hkv;
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
        for (int i = 0; i < R::kN; ++i) to[(4 * i + row) * kBS + slot] = raw[i];
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
            v[(j0 + e) * kBS + slot] = (uint16_t)(u[e / 2] >> (16 * (e % 2)));
        } else {
          uint32_t* v = reinterpret_cast<uint32_t*>(to);
#pragma unroll
          for (int e = 0; e < R::kVec; ++e) v[(j0 + e) * kBS + slot] = u[e];
        }
      }
    }
  }
}

template <int ESZ, int D, int kRot, bool kEven>
static hipError_t launch_qkv_t(const QkvArgs& a) {
  const int heads = a.num_q_heads + 2 * a.num_kv_heads;
  const long long runs = ((long long)a.num_tokens + kBS - 1) / kBS;
  const int per_wave = runs * heads > 16384 ? 4 : 1;
  const int groups = (heads + kQkvWaves * per_wave - 1) / (kQkvWaves * per_wave);
  const long long blocks = runs * groups;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  trace_before(a.stream, "qkv_append");
  hipLaunchKernelGGL((qkv_append_kernel<ESZ, D, kRot, kEven>), dim3((unsigned)blocks),
                     dim3(kQkvWaves * kWave), 0, a.stream, a, groups, per_wave);
  trace_after(a.stream);
  return hipGetLastError();
}

template <int ESZ, int D>
static hipError_t launch_qkv_d(const QkvArgs& a) {
  constexpr int kUnit = 4 * (16 / ESZ);   // rotated dims per register
  if (!a.table) return launch_qkv_t<ESZ, D, 0, false>(a);
#define KV_ROT(N)                                                                     \
  if constexpr (N <= D && N % kUnit == 0)                                             \
    if (a.rot == N)                                                                   \
      return a.interleaved ? launch_qkv_t<ESZ, D, N / kUnit, true>(a)                 \
                           : launch_qkv_t<ESZ, D, N / kUnit, false>(a);
  KV_ROT(32)
  KV_ROT(64)
  KV_ROT(128)
#undef KV_ROT
  return hipErrorNotSupported;
}

hipError_t launch_qkv_append(const QkvArgs& a) {
  if (a.num_tokens == 0) return hipSuccess;
  if (a.head_dim == 128) return a.esz == 2 ? launch_qkv_d<2, 128>(a) : launch_qkv_d<4, 128>(a);
  if (a.head_dim == 64) return a.esz == 2 ? launch_qkv_d<2, 64>(a) : launch_qkv_d<4, 64>(a);
  return hipErrorNotSupported;
}

}  // namespace kvattn
