// Chunked prefill with scores that are capped, biased by distance or cut to a window: the
// tile pipeline of prefill_tile.hpp, with scores made by ModScore.
//
// A tile's steps begin with the block of the first key that its first row sees (window.hpp), so
// that nothing before it is read, and the plan prices items by what is left. The matrix
// work of a step takes a little longer than its softmax beside it, so what a score costs more shows:
//   a window's masks are made only in steps that a window begins in;
//   a bias is one multiply-add in the softmax's own slots (fma(dot, scale, bias - reference));
//   a cap comes before the mask and cannot hide there. Where all of a wavefront's products of a
//     step are under half the cap it is a polynomial of five operations a score, else an
//     exponential, a reciprocal and three more operations.
// A bias or a cap walks a tile's keys from the last to the first: a steep slope's largest
// scores then come first, and the softmax's reference moves once instead of at every step.
// Each kind of scores has kernels of its own, since one that asks for its kind at every score
// needs more registers than there are and spilled. Per call, plain prefill / window of 1024 /
// bias / cap / cap and bias (32 query heads over 8):
//   8192 rows over 24576                    3429 /  207 / 3278 / 4279 / 4311 us
//   the same over 8 bits                    3386 /  194 / 3289 / 4276 / 4259 us
//   4096 rows over 12288                     884 /  106 /  854 / 1102 / 1096 us
//   201 rows over 6150                      49.3 / 36.7 / 52.5 / 61.7 / 59.4 us
//   2048 rows over 6144 and 64 of 1024 to
//     8192, 8 bits                           360 /   82 /  362 /  437 /  426 us
// (the biased ones gain by the order of the keys: near ones hold a row's largest scores.)
// A narrow window leaves most of a call to what a tile has beside its steps: 8192 rows over
// 24576 take 91, 140, 203 and 573 us under windows of 128, 512, 1024 and 4096, 34, 60, 120 and
// 479 of them matrix work that the rows see. The tile map (10 us) comes first, a tile's start,
// first gathers and output are about 6 us with nothing beside them, and each of a tile's
// wavefronts multiplies all of its steps, masked where its 32 rows see none of one.

#pragma once

#include "prefill_tile.hpp"
#include "scoring.hpp"

namespace kvattn {

__device__ __forceinline__ int first_lane(int x) { return __builtin_amdgcn_readfirstlane(x); }

// One workgroup per (item of the plan, or tile of the tile map without one; kv
// head). kRows: the plan may hold one-row sequences.
template <int G, bool kPow2Blocks, bool kRows, Form kForm>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads),
                          amdgpu_waves_per_eu(2, 2)))
void scored_prompt_kernel(const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
                          int num_blocks, const int* __restrict__ block_table,
                          const int* __restrict__ seq_lens, const int* __restrict__ cu,
                          uint16_t* __restrict__ out, PrefillLaunch l, int total_q,
                          int num_q_heads, int num_kv_heads, int max_blocks, int max_seq_len,
                          ModScore<kForm> score) {
  const int g = blockIdx.x % num_kv_heads;
  const int ti = blockIdx.x / num_kv_heads;
  PrefillItem it;
  if (kRows || l.head) {
    it = l.items[ti];   // the list has room for the whole grid: read beside the count
    if (ti >= l.head->items) return;
    // the same in every lane, which a load through a member of l does not tell the compiler
    it = {first_lane(it.s), first_lane(it.q0), first_lane(it.i0), first_lane(it.i1),
          first_lane(it.slot), first_lane(it.cu0), first_lane(it.n), first_lane(it.L)};
  } else {              // no plan: the tile map's whole tiles
    if (ti >= *l.tile_count) return;
    it = whole_tile(l.tiles, ti, cu, seq_lens, total_q, 32 * kWaves / G,
                    min(max_seq_len, max_blocks * kBS), score.window);
  }
  if (kRows && it.q0 < 0)
    prefill_row<G>(it, g, q, kv, num_blocks, block_table, out, l.row_slots, num_q_heads,
                   num_kv_heads, max_blocks, score);
  else
    prefill_tile<G, kPow2Blocks>(it, g, q, kv, num_blocks, block_table, out, l.slots, num_q_heads,
                                 num_kv_heads, max_blocks, score);
}

template <int G, Form kForm>
static hipError_t launch_prefill_scored_t(const PrefillArgs& a, const PrefillLaunch& l) {
  const bool rows = l.head && (a.num_seqs > 1 || a.total_q_tokens == 1);
  const bool pow2 = (a.num_kv_heads & (a.num_kv_heads - 1)) == 0;
  auto kernel = pow2 ? (rows ? scored_prompt_kernel<G, true, true, kForm>
                             : scored_prompt_kernel<G, true, false, kForm>)
                     : (rows ? scored_prompt_kernel<G, false, true, kForm>
                             : scored_prompt_kernel<G, false, false, kForm>);
  hipLaunchKernelGGL(kernel, dim3(l.blocks), dim3(kThreads), 0, a.stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint8_t*>(a.kv),
                     a.num_blocks, a.block_table, a.seq_lens, a.cu_seqlens_q,
                     static_cast<uint16_t*>(a.out), l, a.total_q_tokens, a.num_q_heads,
                     a.num_kv_heads, a.max_blocks, a.max_seq_len,
                     mod_score<kForm>(a.scale, *a.mods));
  return hipGetLastError();
}

template <Form kForm>
static hipError_t dispatch_prefill_scored(const PrefillArgs& a, const PrefillLaunch& l) {
  switch (a.num_q_heads / a.num_kv_heads) {
    case 1: return launch_prefill_scored_t<1, kForm>(a, l);
    case 2: return launch_prefill_scored_t<2, kForm>(a, l);
    case 4: return launch_prefill_scored_t<4, kForm>(a, l);
    case 8: return launch_prefill_scored_t<8, kForm>(a, l);
    default: return hipErrorNotSupported;
  }
}

}  // namespace kvattn
