// Writing a step's new K/V rows into a cache in 8 bits.
//
// A run is the consecutive tokens of slot_mapping that go to one block (at most 16).
// For each run, kv head and K or V: the least exponent e with
// |x| <= 448 * 2^e over the run's finite values; a run that holds slot 0 begins its
// block anew and takes e, another takes max(e, the block's), and where that is
// larger the block's other codes are scaled by the power of two between the two.
// One wavefront does one of these (a task), so that nothing is shared: the rows
// are read once, 16 bytes a lane, the maximum is a wavefront's, and the codes are
// put in order in a tile in LDS. A whole block (16 tokens) and one that is scaled
// anew leave as a whole tile, 16 bytes a lane; others leave as the bytes
// of their tokens alone.
//
// A workgroup of four wavefronts has the runs that begin in a window of the list.
// A window of 16 tokens is one or two runs of a chunk; the tokens of a
// decode step are a run each, and a window of 2 spreads them over the CUs.

#include "common.hpp"
#include "kv_fp8.hpp"
#include "launch.hpp"

namespace kvattn {

namespace {
constexpr int kBS = 16;
constexpr int kAppendWaves = 4;
constexpr int kSmallTokens = 1024;   // up to here windows of kSmallWindow tokens
constexpr int kSmallWindow = 2, kWindow = 16;

// The byte of token r, dim j in a K or V tile.
__device__ __forceinline__ int k_place(int r, int j) { return (j / 16 * kBS + r) * 16 + j % 16; }
__device__ __forceinline__ int v_place(int r, int j) {
  return j / 64 * 1024 + r / 4 * 256 + j % 16 * 16 + j / 16 % 4 * 4 + r % 4;
}

// |x| as an integer that orders like it; 0 for what is not finite.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0;
}

// The exponent byte of a largest value: |x| <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_byte(uint32_t amax) {
  return min(max((int)((amax + 0x1fffffu) >> 23) - 8, kFp8MinByte), kFp8MaxByte);
}

// Two values over the scale as two codes; a finite value past the largest code
// (there is one where the exponent is at its end) becomes that code, infinities and
// NaN the code of NaN.
__device__ __forceinline__ float saturate(float x, float y) {
  return finite_bits(x) == 0 ? y : fminf(fmaxf(y, -448.f), 448.f);
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(saturate(a, a * inv), saturate(b, b * inv), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(saturate(c, c * inv), saturate(d, d * inv), w, true);
}

// Four codes times a power of two.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, r, true);
}

__device__ __forceinline__ uint32_t wave_umax(uint32_t x) {
  // bits of finite floats >= 0 order like the floats
  return __float_as_uint(wave_max(__uint_as_float(x)));
}
}  // namespace

// ESZ: bytes per element of the new rows (2: bf16, 4: fp32).
template <int ESZ, int D, int kWin>
__global__ __launch_bounds__(kAppendWaves * kWave) void kv_append_fp8_kernel(
    const uint8_t* __restrict__ k_new, const uint8_t* __restrict__ v_new,
    const int* __restrict__ slot_mapping, uint8_t* __restrict__ kv, int num_tokens,
    int num_kv_heads, int capacity) {
  constexpr int kVec = 16 / ESZ;               // elements per load
  constexpr int kCh = D / kVec;                // loads per row
  constexpr int kRows = kWave / kCh;           // rows per load of the wavefront
  constexpr int kLoads = kBS / kRows;          // of a whole run
  constexpr int kTileBytes = kBS * D;
  constexpr int kParts = kTileBytes / (kWave * 16);   // 16-byte pieces per lane of a tile
  __shared__ __attribute__((aligned(16))) uint8_t stage[kAppendWaves][kTileBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x % kWave;
  const int g = blockIdx.x % num_kv_heads;
  const int t0 = blockIdx.x / num_kv_heads * kWin;

  // Slots of tokens t0 - 1 .. t0 + kWin + 14, one per lane; which tokens begin a run.
  const int t = t0 - 1 + lane;
  int slot = -1;
  if (lane < kWin + kBS && t >= 0 && t < num_tokens) slot = slot_mapping[t];
  const int block = (unsigned)slot < (unsigned)capacity ? slot / kBS : -1;
  const int before = __shfl_up(block, 1, kWave);
  const bool first = lane > 0 && lane <= kWin && block >= 0 && (before != block);
  // the runs go on while tokens stay in one block
  const unsigned long long same = __ballot(lane > 0 && block >= 0 && before == block);
  unsigned long long runs = __ballot(first);
  uint8_t* tile = stage[wave];

  for (int task = 0; runs; ++task) {
    const int at = __builtin_ctzll(runs);        // lane of the run's first token
    if (task % 2) runs &= runs - 1;              // K, then V of each run
    if (task % kAppendWaves != wave) continue;
    const bool is_v = task % 2;
    const int n = min(kBS, 1 + (int)__builtin_ctzll(~(same >> (at + 1))));
    const int b = __builtin_amdgcn_readlane(block, at);
    const uint8_t* src = (is_v ? v_new : k_new) +
                         ((size_t)(t0 - 1 + at) * num_kv_heads + g) * (D * ESZ);
    uint8_t* base = kv + (size_t)b * fp8_block_bytes(num_kv_heads, D);
    uint8_t* dst = base + (size_t)((is_v ? num_kv_heads : 0) + g) * kTileBytes;
    uint8_t* exp = base + fp8_tiles_bytes(num_kv_heads, D) + 2 * g + is_v;
    const int old = *exp;

    // ---- the run's rows, and their largest value ----
    const int sub = lane / kCh, ch = lane % kCh;
    uint4 x[kLoads];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = i * kRows + sub;
      x[i] = make_uint4(0, 0, 0, 0);
      if (row < n)
        x[i] = *reinterpret_cast<const uint4*>(src + (size_t)row * num_kv_heads * (D * ESZ) + ch * 16);
    }
    auto value = [&](int i, int e) __attribute__((always_inline)) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      if constexpr (ESZ == 2) return e % 2 ? bf16hi(w[e / 2]) : bf16lo(w[e / 2]);
      else return __uint_as_float(w[e]);
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e) amax = max(amax, finite_bits(value(i, e)));
    amax = wave_umax(amax);

    // ---- the block's exponent ----
    const unsigned long long mine = ((1ull << n) - 1) << at;
    const bool fresh = (__ballot(slot % kBS == 0) & mine) != 0;
    const int kept = min(max(old, kFp8MinByte), kFp8MaxByte);
    const int need = exponent_byte(amax);
    const int byte = fresh ? need : max(kept, need);
    const bool grown = !fresh && byte != kept;
    // 16 powers of two add up to 2^16 - 1 only if they are all different ones
    const bool in_run = lane >= at && lane < at + n;
    const bool whole = wave_sum(in_run ? (float)(1 << (slot & 15)) : 0.f) == 65535.f && n == kBS;
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
    const float inv = fp8_scale(254 - byte);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = i * kRows + sub;
      const int r = __shfl(slot, at + min(row, n - 1), kWave) % kBS;
      if (row >= n) continue;
      const int j = ch * kVec;
      uint32_t w[kVec / 4];
#pragma unroll
      for (int c = 0; c < kVec / 4; ++c)
        w[c] = encode4(value(i, 4 * c), value(i, 4 * c + 1), value(i, 4 * c + 2),
                       value(i, 4 * c + 3), inv);
      if (!is_v) {
#pragma unroll
        for (int c = 0; c < kVec / 4; ++c)
          *reinterpret_cast<uint32_t*>(to + k_place(r, j + 4 * c)) = w[c];
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) to[v_place(r, j + e)] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
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

template <int ESZ, int D>
static hipError_t launch_append_fp8_t(const AppendArgs& a) {
  const bool small = a.num_tokens <= kSmallTokens;
  const int win = small ? kSmallWindow : kWindow;
  const long long blocks = ((long long)a.num_tokens + win - 1) / win * a.num_kv_heads;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  auto kernel = small ? kv_append_fp8_kernel<ESZ, D, kSmallWindow>
                      : kv_append_fp8_kernel<ESZ, D, kWindow>;
  trace_before(a.stream, "kv_append_fp8");
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kAppendWaves * kWave), 0, a.stream,
                     static_cast<const uint8_t*>(a.k_new), static_cast<const uint8_t*>(a.v_new),
                     a.slot_mapping, static_cast<uint8_t*>(a.kv), a.num_tokens, a.num_kv_heads,
                     a.num_blocks * kBS);
  trace_after(a.stream);
  return hipGetLastError();
}

hipError_t launch_append_fp8(const AppendArgs& a) {
  if (a.head_dim == 128)
    return a.esz == 2 ? launch_append_fp8_t<2, 128>(a) : launch_append_fp8_t<4, 128>(a);
  if (a.head_dim == 64)
    return a.esz == 2 ? launch_append_fp8_t<2, 64>(a) : launch_append_fp8_t<4, 64>(a);
  return hipErrorNotSupported;
}

}  // namespace kvattn
