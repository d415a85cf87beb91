// What a step's calls read, from the requests' lengths: how many of each request's
// new tokens the step takes, the new blocks they need, handed out of a list of
// free ids in order, and the slot and position of every token.
//
// For request s with c_s cached tokens, w_s wanted ones and a table of C tokens:
//   n_s  = min(max(w_s, 0), C - c_s), then in order until max_tokens are taken:
//   cu_s = min(sum of n over requests before s, max_tokens), n_s = cu_(s+1) - cu_s
//   new entries of its table: [ceil(c_s / 16), ceil((c_s + n_s) / 16)), the ids
//   from place sum over requests before s of their count
// Two sums over the requests, one after the other since the second counts what
// the first has cut; the first saturates at max_tokens, which is associative and stays
// below 32 bits. Bound by latency: one launch, in which every workgroup does the
// sums for itself (requests in tiles, one tile in nearly every call)
// and then writes its share of the tile's requests and tokens, finding a token's
// request by a search in LDS. A thread per token, in up to 64 workgroups: 2048 requests
// with 24 prompts and 16384 tokens took 11.1 / 9.2 / 7.9 us at 4 / 2 / 1 tokens a
// thread, 7.0 with workgroups of 512 threads instead of 1024, and 5.4 without reading
// the partial blocks' ids ahead for all requests (rocprof). 256 requests of one token
// each take 3.5 us with 256 threads (5.9 with 1024); an empty kernel takes about 2.

#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace kvattn {

namespace {
constexpr int kBS = 16;
constexpr int kPer = 4;                    // requests per thread and tile
constexpr int kFewThreads = 256, kManyThreads = 512;
constexpr int kMostGroups = 64;            // workgroups per tile

// Sums over the lanes up to this one, at most cap; x and cap below 2^31. Four steps within
// rows of 16 lanes, then each row's total to the rows behind it.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t scan_step(uint32_t x, uint32_t cap) {
  return min(x + (uint32_t)__builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xf, false), cap);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, uint32_t cap) {
  x = scan_step<0x111, 0xf>(x, cap);   // row_shr 1, 2, 4, 8
  x = scan_step<0x112, 0xf>(x, cap);
  x = scan_step<0x114, 0xf>(x, cap);
  x = scan_step<0x118, 0xf>(x, cap);
  x = scan_step<0x142, 0xa>(x, cap);   // row_bcast 15 into rows 1 and 3
  return scan_step<0x143, 0xc>(x, cap);   // row_bcast 31 into rows 2 and 3
}

// The sum over the threads before this one, and over all, at most cap.
template <int kThreads>
__device__ __forceinline__ uint32_t group_scan(uint32_t v, uint32_t cap, uint32_t* lds,
                                               uint32_t* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t x = wave_scan(v, cap);
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) {
    const uint32_t y = lds[w];
    before = min(before + (w < wave ? y : 0), cap);
    all = min(all + y, cap);
  }
  __syncthreads();
  *total = all;
  const uint32_t left = __shfl_up(x, 1, kWave);
  return lane ? min(before + left, cap) : before;
}
}  // namespace

template <int kThreads>
__global__ __launch_bounds__(kThreads) void step_map_kernel(StepMapArgs a, int tiles, int groups) {
  constexpr int kTile = kThreads * kPer;
  __shared__ int cu[kTile + 1], cached[kTile], ids_at[kTile];
  __shared__ uint32_t scan[kThreads / kWave];
  const int tid = threadIdx.x;
  const int my_tile = blockIdx.x / groups, group = blockIdx.x % groups;
  const int room = a.max_blocks * kBS;
  const uint32_t most = a.max_tokens;
  constexpr uint32_t kNoCap = 0x7fffffff;
  uint32_t tokens = 0, ids = 0;                  // of the tiles before
  int base = 0;
  for (int tile = 0;; ++tile) {
    base = tile * kTile;
    int c[kPer], held[kPer], own[kPer];
    uint32_t n[kPer], sum = 0, total;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int s = base + k * kThreads + tid;   // coalesced; by thread from LDS below
      c[k] = s < a.num_seqs ? max(a.cached[s], 0) : 0;
      const int w = s < a.num_seqs ? a.wanted[s] : 0;
      cu[k * kThreads + tid] = min(max(w, 0), max(room - c[k], 0));
      cached[k * kThreads + tid] = c[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      c[k] = cached[tid * kPer + k];
      held[k] = (int)(((uint32_t)c[k] + kBS - 1) / kBS);
      n[k] = min((uint32_t)cu[tid * kPer + k], most);
      sum = min(sum + n[k], most);
    }
    uint32_t at = min(tokens + group_scan<kThreads>(sum, most, scan, &total), most);
    tokens = min(tokens + total, most);
    uint32_t new_ids = 0, first[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      first[k] = at;
      at = min(at + n[k], most);
      own[k] = (int)(((uint32_t)c[k] + (at - first[k]) + kBS - 1) / kBS) - held[k];
      new_ids += own[k];
    }
    uint32_t id_at = ids + group_scan<kThreads>(new_ids, kNoCap, scan, &total);
    ids += total;
    if (tile < my_tile) continue;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = tid * kPer + k;
      cu[i] = first[k];
      ids_at[i] = id_at;
      id_at += own[k];
    }
    if (tid == 0) cu[kTile] = tokens;
    break;
  }
  __syncthreads();

  // ---- the tile's requests ----
  const int here = min(kTile, a.num_seqs - base);
  for (int i = group * kThreads + tid; i < here; i += groups * kThreads) {
    a.seq_lens[base + i] = cached[i] + cu[i + 1] - cu[i];
    a.cu_seqlens_q[base + i] = cu[i];
  }
  const int end = cu[kTile];
  const bool last = my_tile == tiles - 1;
  if (last && group == 0 && tid == 0) {
    a.cu_seqlens_q[a.num_seqs] = end;
    a.used[0] = end;
    a.used[1] = ids;
  }

  // ---- its tokens; the first token of a new block writes the block's entry ----
  const int stride = groups * kThreads;
  for (long long tl = (long long)cu[0] + group * kThreads + tid; tl < end; tl += stride) {
    const int t = (int)tl;
    int lo = 0, hi = here - 1;                   // last request with cu <= t: it has t
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (cu[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int pos = cached[lo] + t - cu[lo];
    const int held = (int)(((uint32_t)cached[lo] + kBS - 1) / kBS);
    const int entry = pos / kBS;
    int* row = a.block_table + (size_t)(base + lo) * a.max_blocks;
    int id;
    if (entry < held) {   // the partial block the request holds
      id = row[entry];
    } else {
      const uint32_t place = (uint32_t)ids_at[lo] + entry - held;
      id = place < (uint32_t)a.num_free ? a.free_ids[place] : -1;
      if (pos % kBS == 0) row[entry] = id;
    }
    a.slot_mapping[t] = id >= 0 && id <= (0x7fffffff - (kBS - 1)) / kBS ? id * kBS + pos % kBS : -1;
    a.positions[t] = pos;
  }
  // ---- rows of the step that no token has ----
  if (!last) return;
  for (long long t = (long long)end + group * kThreads + tid; t < a.max_tokens; t += stride) {
    a.slot_mapping[t] = -1;
    a.positions[t] = 0;
  }
}

template <int kThreads>
static void launch_step_map_t(const StepMapArgs& a) {
  constexpr int kTile = kThreads * kPer;
  const int tiles = std::max(1, (a.num_seqs + kTile - 1) / kTile);
  const int groups =
      std::min(kMostGroups, std::max(1, (int)(((long long)a.max_tokens + kThreads - 1) /
                                              kThreads)));
  hipLaunchKernelGGL(step_map_kernel<kThreads>, dim3(tiles * groups), dim3(kThreads), 0, a.stream,
                     a, tiles, groups);
}

hipError_t launch_step_map(const StepMapArgs& a) {
  trace_before(a.stream, "step_map");
  if (a.num_seqs <= kFewThreads * kPer)
    launch_step_map_t<kFewThreads>(a);
  else
    launch_step_map_t<kManyThreads>(a);
  trace_after(a.stream);
  return hipGetLastError();
}

}  // namespace kvattn
