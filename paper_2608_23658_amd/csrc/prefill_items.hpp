// What the chunked-prefill kernels of the two cache formats share: work items and
// where their partials lie, and the device helpers of the tile pipelines.
#pragma once

#include "common.hpp"
#include "window.hpp"

namespace kvattn {

namespace {

constexpr int kD = 128;
constexpr int kBS = 16;
constexpr int kKeys = 64;                  // keys per step
constexpr int kStepBlocks = 4;             // blocks per step
constexpr float kLazyRescale = 8.f;        // log2 headroom before the max moves
constexpr float kPsumBound = 256.f;         // 2^kLazyRescale
constexpr int kWaves = 8;                  // wavefronts per workgroup
constexpr int kThreads = kWaves * kWave;
constexpr int kNumCUs = 256;               // gfx950
static_assert(kBS == 16 && kKeys == 64, "as window.hpp takes them");

typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16_t mfma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// max(a, b, c) in one instruction. The scores here are never NaN (masked
// keys are set to -inf by a select), so the IEEE NaN handling that fmaxf
// adds around every operand is not needed.
__device__ __forceinline__ float max3f(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// Two loads of 16 bytes per lane from global memory straight into LDS
// (global_load_lds_dwordx4): load j has lane l read base_j + off_j and its
// bytes land at LDS byte address lds_j + 16 l (base_j and lds_j wave-uniform,
// in SGPRs). A wave-uniform base plus a 32-bit lane offset takes the address
// unit fewer cycles per instruction than 64 lanes of 64-bit addresses. M0
// carries each load's LDS address: the block saves the compiler's M0 first
// and restores it last, so no code outside the block sees M0 change. Issued
// as inline assembly so that the compiler does not treat the loads as LDS
// stores that every later LDS read must wait for: the callers wait for them
// themselves (s_waitcnt vmcnt) before the barrier that publishes the data.
__device__ __forceinline__ void dma16x2(const void* base0, uint32_t off0, uint32_t lds0,
                                        const void* base1, uint32_t off1, uint32_t lds1) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2\n\t"
      "s_mov_b32 m0, %6\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %4, %5\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(off0), "s"(base0), "s"(lds0), "v"(off1), "s"(base1), "s"(lds1)
      : "memory");
}

// Entry i of a block-table row, read by a scalar memory load: the row pointer
// is wave-uniform and the index is made so, and a load through the constant
// address space from a uniform address is a scalar load. It is therefore
// counted by lgkmcnt, never by the vmcnt that the gathers are waited with.
__device__ __forceinline__ int scalar_entry(const int* row, int i) {
  const __attribute__((address_space(4))) int* p =
      (const __attribute__((address_space(4))) int*)row;
  return p[(unsigned)__builtin_amdgcn_readfirstlane(i)];
}

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef i32x4_t i32x4_a4_t __attribute__((aligned(4)));

// Entries i .. i + 3 of a block-table row in one 16-byte scalar load (scalar
// loads need only 4-byte alignment).
__device__ __forceinline__ i32x4_t scalar_entries4(const int* row, int i) {
  const __attribute__((address_space(4))) i32x4_a4_t* p =
      (const __attribute__((address_space(4))) i32x4_a4_t*)(
          row + (unsigned)__builtin_amdgcn_readfirstlane(i));
  return *p;
}

// LDS byte address of a pointer into a __shared__ array.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// The lane's index in its wavefront, computed afresh at each call (volatile,
// so it is not merged with an earlier copy that would have to stay live).
__device__ __forceinline__ int lane_id_fresh() {
  int r;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(r));
  return r;
}

}  // namespace

// Rows [lo, hi) of sequence s's chunk, with the offsets clamped into
// [0, total_q] and hi >= lo, so that offsets that break the documented
// contract (decreasing, or past the end of q) can neither read nor write
// outside q and out.
__device__ __forceinline__ int2 chunk_rows(const int* __restrict__ cu, int s, int total_q) {
  const int lo = min(max(cu[s], 0), total_q);
  const int hi = min(max(cu[s + 1], lo), total_q);
  return make_int2(lo, hi);
}

struct PrefillItem {
  int s, q0;        // sequence, first row of the tile in the chunk (-1: one-row item)
  int i0, i1;       // key steps from the tile's walk_start on, i0 even (one-row item: tokens,
                    // i0 a multiple of 16)
  int slot;         // partial slot, -1: written to out
  int cu0, n, L;    // the sequence's chunk and clamped length
};

// The item of workgroup (ti, kv head) of a launch without a plan: tile ti of the tile map.
__device__ __forceinline__ PrefillItem whole_tile(const int2* __restrict__ tiles, int ti,
                                                  const int* __restrict__ cu,
                                                  const int* __restrict__ seq_lens, int total_q,
                                                  int rows_per_tile, int max_tokens, int window) {
  PrefillItem it;
  const int2 tl = tiles[ti];
  const int2 rows = chunk_rows(cu, tl.x, total_q);
  it.s = tl.x;
  it.q0 = tl.y;
  it.cu0 = rows.x;
  it.n = rows.y - rows.x;
  it.L = min(max(seq_lens[tl.x], 0), max_tokens);
  const int pos = it.L - it.n + it.q0;
  it.i0 = 0;
  it.i1 = walk_steps(pos, min(pos + min(rows_per_tile, it.n - it.q0) - 1, it.L - 1), window);
  it.slot = -1;
  return it;
}

struct PrefillPlan {
  int items, splits, row_splits, pad;
};

// A slot holds, for each of the 8 wavefronts of a tile and its 32 rows, O
// unnormalised in fp32 as [dim pair][row] and (reference max, row sum).
constexpr int kSlotFloats = kWaves * 32 * kD;
constexpr size_t kSlotBytes = kSlotFloats * sizeof(float) + kWaves * 32 * sizeof(float2);

// A one-row slot: O [G][kD] and (max, row sum) [G], whole 16 bytes.
constexpr size_t row_slot_bytes(int group) {
  return ((size_t)group * (kD * sizeof(float) + sizeof(float2)) + 15) & ~size_t(15);
}

}  // namespace kvattn
