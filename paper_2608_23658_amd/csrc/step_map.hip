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
// the first has cut. Bound by latency: one launch, in which every workgroup does the
// sums for itself (requests in tiles of 4096, one tile in nearly every call)
// and then writes its share of the tile's requests and tokens, finding a
// token's request by a search in LDS.

#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace kvattn {

namespace {
constexpr int kBS = 16;
constexpr int kMapThreads = 1024;
constexpr int kPer = 4;                          // requests per thread and tile
constexpr int kMapTile = kMapThreads * kPer;
constexpr int kTokensPerGroup = 2048;            // tokens for which a workgroup is added
constexpr int kMostGroups = 64;                  // per tile

// Exclusive sum over the workgroup of one value per thread, and the total.
__device__ __forceinline__ long long group_scan(long long v, long long* lds, long long* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  long long x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long long y = __shfl_up(x, o, kWave);
    x += lane >= o ? y : 0;
  }
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMapThreads / kWave; ++w) {
    before += w < wave ? lds[w] : 0;
    all += lds[w];
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}
}  // namespace

__global__ __launch_bounds__(kMapThreads) void step_map_kernel(StepMapArgs a, int tiles,
                                                               int groups) {
  __shared__ int cu[kMapTile + 1], cached[kMapTile], ids_at[kMapTile];
  __shared__ long long scan[kMapThreads / kWave];
  const int tid = threadIdx.x;
  const int my_tile = blockIdx.x / groups, group = blockIdx.x % groups;
  const long long room = (long long)a.max_blocks * kBS;
  long long tokens = 0, ids = 0;                 // of the tiles before
  int base = 0;
  for (int tile = 0;; ++tile) {
    base = tile * kMapTile;
    int c[kPer];
    long long n[kPer], sum = 0, total;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int s = base + tid * kPer + k;
      c[k] = s < a.num_seqs ? max(a.cached[s], 0) : 0;
      const int w = s < a.num_seqs ? a.wanted[s] : 0;
      n[k] = max(min((long long)max(w, 0), room - c[k]), 0ll);
      sum += n[k];
    }
    long long at = tokens + group_scan(sum, scan, &total);
    int new_ids = 0;
    int first[kPer], took[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      first[k] = (int)min(at, (long long)a.max_tokens);
      at += n[k];
      took[k] = (int)min(at, (long long)a.max_tokens) - first[k];
      new_ids += (int)(((long long)c[k] + took[k] + kBS - 1) / kBS - ((long long)c[k] + kBS - 1) / kBS);
    }
    tokens += total;
    long long id_at = ids + group_scan(new_ids, scan, &total);
    ids += total;
    if (tile < my_tile) continue;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = tid * kPer + k;
      cu[i] = first[k];
      cached[i] = c[k];
      ids_at[i] = (int)min(id_at, (long long)0x7fffffff);
      id_at += ((long long)c[k] + took[k] + kBS - 1) / kBS - ((long long)c[k] + kBS - 1) / kBS;
    }
    if (tid == 0) cu[kMapTile] = (int)min(tokens, (long long)a.max_tokens);
    break;
  }
  __syncthreads();

  // ---- the tile's requests ----
  const int here = min(kMapTile, a.num_seqs - base);
  for (int i = group * kMapThreads + tid; i < here; i += groups * kMapThreads) {
    a.seq_lens[base + i] = cached[i] + cu[i + 1] - cu[i];
    a.cu_seqlens_q[base + i] = cu[i];
  }
  const int end = cu[kMapTile];
  const bool last = my_tile == tiles - 1;
  if (last && group == 0 && tid == 0) {
    a.cu_seqlens_q[a.num_seqs] = end;
    a.used[0] = end;
    a.used[1] = (int)min(ids, (long long)0x7fffffff);
  }

  // ---- its tokens; the first token of a new block writes the block's entry ----
  const int stride = groups * kMapThreads;
  for (int t = cu[0] + group * kMapThreads + tid; t < end; t += stride) {
    int lo = 0, hi = here - 1;                   // last request with cu <= t: it has t
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (cu[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int pos = cached[lo] + t - cu[lo];
    const int held = (int)(((long long)cached[lo] + kBS - 1) / kBS);
    const int entry = pos / kBS;
    int* row = a.block_table + (size_t)(base + lo) * a.max_blocks;
    int id;
    if (entry < held) {
      id = row[entry];
    } else {
      const long long place = (long long)ids_at[lo] + entry - held;
      id = place < a.num_free ? a.free_ids[place] : -1;
      if (pos % kBS == 0) row[entry] = id;
    }
    a.slot_mapping[t] = id >= 0 && id <= (0x7fffffff - (kBS - 1)) / kBS ? id * kBS + pos % kBS : -1;
    a.positions[t] = pos;
  }
  // ---- rows of the step that no token has ----
  if (!last) return;
  for (long long t = (long long)end + group * kMapThreads + tid; t < a.max_tokens; t += stride) {
    a.slot_mapping[t] = -1;
    a.positions[t] = 0;
  }
}

hipError_t launch_step_map(const StepMapArgs& a) {
  const int tiles = std::max(1, (a.num_seqs + kMapTile - 1) / kMapTile);
  const int groups =
      std::min(kMostGroups, std::max(1, (a.max_tokens + kTokensPerGroup - 1) / kTokensPerGroup));
  trace_before(a.stream, "step_map");
  hipLaunchKernelGGL(step_map_kernel, dim3(tiles * groups), dim3(kMapThreads), 0, a.stream, a, tiles,
                     groups);
  trace_after(a.stream);
  return hipGetLastError();
}

}  // namespace kvattn
