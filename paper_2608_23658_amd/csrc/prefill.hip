// Chunked-prefill attention for gfx950 on bf16 MFMA (the paper, Section 5:
// prefill is compute bound and a chunk attends to all earlier context, so
// chunking splits the same work; Section 1: max_num_batched_tokens bounds
// the chunk).
//
// Here the plan of a step, the merge of shared tiles and the launches; prefill_tile.hpp has
// the work of a tile.

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "decode_walk.hpp"
#include "launch.hpp"
#include "prefill_items.hpp"
#include "prefill_tile.hpp"
#include "scoring.hpp"

namespace kvattn {

// Lists the work tiles (sequence, first row) of a batch of chunks, the rows
// of a sequence's chunk in descending order so the longest rows start first.
__global__ __launch_bounds__(256) void prefill_tile_map_kernel(const int* __restrict__ cu,
                                                               int num_seqs, int total_q,
                                                               int rows_per_tile,
                                                               int2* __restrict__ tiles,
                                                               int* __restrict__ count,
                                                               int max_tiles) {
  __shared__ int scan[256];
  const int tid = threadIdx.x;
  const int per = (num_seqs + 255) / 256;
  const int s0 = min(num_seqs, tid * per);
  const int s1 = min(num_seqs, s0 + per);
  int mine = 0;
  for (int s = s0; s < s1; ++s) {
    const int2 r = chunk_rows(cu, s, total_q);
    mine += (r.y - r.x + rows_per_tile - 1) / rows_per_tile;
  }
  scan[tid] = mine;
  __syncthreads();
  for (int o = 1; o < 256; o <<= 1) {
    const int v = tid >= o ? scan[tid - o] : 0;
    __syncthreads();
    scan[tid] += v;
    __syncthreads();
  }
  int off = scan[tid] - mine;
  for (int s = s0; s < s1; ++s) {
    const int2 r = chunk_rows(cu, s, total_q);
    const int nt = (r.y - r.x + rows_per_tile - 1) / rows_per_tile;
    for (int k = 0; k < nt; ++k) {
      if (off < max_tiles) tiles[off] = make_int2(s, (nt - 1 - k) * rows_per_tile);
      ++off;
    }
  }
  if (tid == 255) *count = min(scan[255], max_tiles);
}

// ---- planned steps ----
//
// With the workspace kvattn_prefill_workspace_bytes asks for, a step's work is
// laid out by a plan kernel. An item is a run of key steps of one work tile
// (for all kv heads); a tile whose keys are shared by several items leaves a
// partial state per item in a slot, and prefill_combine_kernel merges them.
// A tile is a serial walk of about 1.7 us per key step, one workgroup per CU,
// so a step with few tiles leaves CUs idle, and one whose tiles do not divide
// by the CUs idles them in its last round. A call at 32 query heads over 8,
// whole tiles in sequence order against planned items:
//   201 rows over 6150 cached tokens (32 workgroups of 100 steps)  162 -> 44 us
//   512 rows over 8192                                             215 -> 88 us
//   1024 rows over 1024                                             62 -> 53 us
//   9 chunks of 100 to 900 rows over 1000 to 8000 tokens           443 -> 367 us
//   8192 rows over 24576 (four even rounds, not shared)           3274, 3278 us
// Items go by length over all sequences. Of 15 steps of 3 to 20 chunks that share
// nothing, 13 gain up to 11% by it against sequence by sequence or stay, and two of
// sequences alike lose 5%: 9 chunks of 300 to 600 rows over 1500 to 3000 tokens, 64
// query heads over 8, 306 -> 323 us, 9 of 113 to 679 over 1722 to 3445 275 -> 289.
// Coarser lengths (8 or 32 classes instead of 256) give 2% back on the first and
// lose up to 3% on others.
//
// A sequence that adds one row (a decode sequence in a unified step) is no tile:
// its tile would put one row of each head through 32-row products and stage its
// whole context through LDS for them. It takes decode's walk instead, a
// workgroup's eight wavefronts sharing an item's tokens. Such items are bound by
// HBM and tiles by the matrix units, so the plan lets them run side by side. A
// call at 32 query heads over 8, one-row sequences as tiles against this:
//   2048 rows over 6144 cached tokens, 128 one-row of 1024 to 8192   645 -> 435 us
//   8192 rows over 24576, the same 128                             3667 -> 3477 us
//   two chunks of 5 and 9 rows, 100 one-row of 1024 to 8192          371 -> 306 us
//   64 query heads: 512 rows over 1000, 40 one-row of 1024 to 8192   268 -> 142 us

struct PrefillSplit {   // a tile shared by several items
  int row0, rows;       // its rows in q and out
  int slot0, pieces;
};

struct RowSplit {       // a one-row sequence shared by several items
  int row, slot0, pieces, pad;
};

constexpr int kPlanThreads = 512;
constexpr int kPlanCandidates = 16;
// Estimated cost, in key steps, of an item's prologue and epilogue, and of
// writing and merging a partial.
constexpr int kItemSteps = 3, kPartialSteps = 6;
// A one-row item's time per 64 tokens and kv head, in key steps: on its CU
// (eight wavefronts, a step of about 2 us each), and of the whole chip's HBM
// time (32 KiB at 4.6 TB/s: the tiles beside it read too). 2048 rows over 6144
// cached tokens with 128 one-row sequences of 1024 to 8192: 502 / 443 / 435 /
// 502 us at 0.15 / 0.3 / 0.5 / 0.8 with the HBM term at 0.0031, and 441 / 439 /
// 430 / 438 us at 0.0015 / 0.0031 / 0.0045 / 0.006; 512 rows over 1000 with 40
// of them 141 / 141 / 149 / 150 us and 141 / 141 / 143 / 143.
constexpr float kRowStep = 0.3f, kRowHbmStep = 0.0042f;
constexpr int kRowTokens = 1024;   // fewest tokens of a shared sequence's item
constexpr int kCombineParts = 4;   // workgroups over the dims of a merge
constexpr int kCombineGrid = 1024;

struct PlanArgs {
  const int* cu;
  const int* seq_lens;
  int num_seqs, total_q, rows_per_tile, num_kv_heads, max_seq_tokens;
  int max_items, max_slots;   // max_slots 0: no tile is shared
  int rows, max_row_slots;    // rows 0: one-row sequences are tiles
  int window;                 // keys a row sees, kNoWindow: all up to its own
  PrefillItem* items;
  PrefillSplit* splits;
  RowSplit* row_splits;
  PrefillPlan* head;
};

// Whether sharing tiles can gain more than it costs, for a call whose longest
// tile walks this many key steps and whose tiles are this many workgroups: below
// eight steps an item's own cost outweighs what it saves, four or more rounds of
// tiles gain nothing, and up to 64 steps the longest walk, over the part of the
// last round that is idle, has to be min_steps. The host asks with its bounds
// whether the wider plan and the merge are worth a launch. 32 query heads over 8,
// whole tiles, shared, and not shared by that rule:
//   2 of 770 rows over 50                         36 / 38 / 33 us
//   9 of 176 over 692, with 2 one-row             38 / 46 / 35 us
//   440 rows over 227                             29 / 31 / 27 us
// and shared by it: 53 -> 41 us (1673 rows with 15 one-row, 8 query heads over 8).
// With a loose bound it launches them, and the plan asks whether to weigh
// candidates, with the lengths. Not shared / shared, under a bound of 131072 (the
// longest walk over the idle part): 512 rows over 256 (9.0) 29.8 / 32.2 us, 200
// over 512 (10.5) 28.5 / 27.1, 1024 over 256 (10.0) 41.9 / 39.5, 1024 over 1024
// (16.0) 59.3 / 53.3.
constexpr int kLaunchSteps = 16, kPlanSteps = 10;
__host__ __device__ __forceinline__ bool sharing_pays(long long steps, long long workgroups,
                                                      int min_steps) {
  const long long chip = workgroups > kNumCUs ? (workgroups + kNumCUs - 1) / kNumCUs * kNumCUs
                                              : kNumCUs;
  return steps > 8 && workgroups < 4 * kNumCUs &&
         (steps > 64 || steps * (chip - workgroups) >= min_steps * chip);
}

// Steps per item and items of a tile of N steps, at most C steps per item.
__device__ __forceinline__ int2 tile_pieces(int N, int C) {
  const int p = (N - 1) / C + 1;
  if (N <= 0 || p <= 1) return make_int2(max(N, 0), 1);
  const int per = (((N + p - 1) / p) + 1) & ~1;   // whole pairs of steps
  return make_int2(per, (N + per - 1) / per);
}

// Tokens per item and items of a one-row sequence of L tokens, at most C
// tokens (a multiple of 64) per item.
__device__ __forceinline__ int2 row_pieces(int L, int C) {
  const int p = (L - 1) / C + 1;
  if (L <= 0 || p <= 1) return make_int2(max(L, 0), 1);
  const int per = ((L - 1) / p / kKeys + 1) * kKeys;
  return make_int2(per, (L - 1) / per + 1);
}

// Exclusive prefix sums of v and of flag over the workgroup, and their totals.
struct PlanScan {
  int before, total, set_before, set_total;
};
__device__ __forceinline__ PlanScan plan_scan(int v, bool flag, int2* lds) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o, kWave);
    x += lane >= o ? y : 0;
  }
  const unsigned long long set = __ballot(flag);
  if (lane == kWave - 1) lds[wave] = make_int2(x, (int)__popcll(set));
  __syncthreads();
  PlanScan r = {x - v, 0, (int)__popcll(set & ((1ull << lane) - 1)), 0};
#pragma unroll
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    const int2 e = lds[w];
    r.before += w < wave ? e.x : 0;
    r.total += e.x;
    r.set_before += w < wave ? e.y : 0;
    r.set_total += e.y;
  }
  __syncthreads();
  r.total = __builtin_amdgcn_readfirstlane(r.total);
  r.set_total = __builtin_amdgcn_readfirstlane(r.set_total);
  return r;
}

// Sums and maxima over the workgroup, in one order whatever the timing: a
// wavefront's by its fixed tree, then the wavefronts' one after another.
struct PlanTotals {
  float steps, tokens;           // sums: they only feed estimates
  float max_steps, max_tokens;
};
__device__ __forceinline__ PlanTotals plan_totals(PlanTotals v, PlanTotals* lds) {
  v = {wave_sum(v.steps), wave_sum(v.tokens), wave_max(v.max_steps), wave_max(v.max_tokens)};
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  PlanTotals r = lds[0];
#pragma unroll
  for (int w = 1; w < kPlanThreads / kWave; ++w) {
    const PlanTotals e = lds[w];
    r = {r.steps + e.steps, r.tokens + e.tokens, fmaxf(r.max_steps, e.max_steps),
         fmaxf(r.max_tokens, e.max_tokens)};
  }
  return r;
}

// Tile t of a chunk of sequences: its sequence's index in the chunk, first row,
// key steps.
struct PlanTile {
  int idx, q0, steps;
};

struct PlanChoice {
  int limit, x, y;              // steps per item; CUs / kv heads for tiles, for one-row items
  float tile_time, row_time;    // a tile item's time; a one-row item's on its CU
};

// Latency-bound, one workgroup ahead of the attention kernel. kResident: the
// sequences fit one chunk (512) and their tiles one per thread, the usual case,
// and each thread keeps its tile in registers over all passes. A call that runs in
// one round needs no order and is written at once, also with one-row sequences: 2.5
// us (rocprof), as the tile map. Ordering takes 5.4, candidates to weigh or one-row
// sequences to mix in 7.1, both 10.0. A call of 143 rows with 16 one-row sequences
// under 814 tokens, 8 query heads over 8, took 23.8 us with the ordering passes and
// takes 19.8, 9 of 176 over 692 with 2, 32 over 8, 39.5 and 35.0.
template <bool kResident>
__global__ __launch_bounds__(kPlanThreads) void prefill_plan_kernel(PlanArgs args) {
  __shared__ int seq_cu[kPlanThreads], seq_n[kPlanThreads], seq_L[kPlanThreads];
  __shared__ int first[kPlanThreads + 1];     // first tile of each sequence of the chunk
  __shared__ int2 scan_lds[kPlanThreads / kWave];
  __shared__ int hist[256], row_hist[256], steps[kPlanThreads];
  __shared__ PlanTotals totals_lds[kPlanThreads / kWave];
  __shared__ int extra_row_items, next_slot, next_split, next_row_slot, next_row_split,
      row_slots_needed;
  __shared__ int cand_items[kPlanCandidates], cand_slots[kPlanCandidates];
  __shared__ PlanChoice choice;
  const int tid = threadIdx.x;
  PlanArgs a = args;
  if constexpr (!kResident) {
    // kept in vector registers: the nested loops leave too few scalar ones
    __shared__ PlanArgs lds_args;
    if (tid == 0) lds_args = args;
    __syncthreads();
    a = lds_args;
    a.num_seqs = args.num_seqs;   // the bound of the loops with barriers stays uniform
  }
  const int R = a.rows_per_tile;
  const int seqs = min(a.num_seqs, kPlanThreads);   // sequences of a chunk, at most

  // Loads sequences base .. base + 511 and numbers their tiles.
  auto load_chunk = [&](int base) {
    const int s = base + tid;
    int nt = 0;
    bool row = false;
    if (s < a.num_seqs) {
      const int len = a.seq_lens[s];
      const int2 r = chunk_rows(a.cu, s, a.total_q);
      seq_cu[tid] = r.x;
      seq_n[tid] = r.y - r.x;
      seq_L[tid] = min(max(len, 0), a.max_seq_tokens);
      row = a.rows && r.y - r.x == 1;
      nt = row ? 0 : (r.y - r.x + R - 1) / R;
    }
    const PlanScan at = plan_scan(nt, row, scan_lds);
    first[tid] = at.before;
    if (tid == 0) first[kPlanThreads] = at.total;
    __syncthreads();
    return at;   // of tiles and one-row sequences
  };
  // The rows of a sequence are taken in descending order.
  auto tile_of = [&](int t) {
    int lo = 0, hi = seqs - 1;   // last sequence with first <= t, which has tiles
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (first[mid] <= t) lo = mid; else hi = mid - 1;
    }
    PlanTile r;
    const int nt = (lo + 1 < kPlanThreads ? first[lo + 1] : first[kPlanThreads]) - first[lo];
    const int n = seq_n[lo], L = seq_L[lo];
    r.idx = lo;
    r.q0 = (nt - 1 - (t - first[lo])) * R;
    const int pos = L - n + r.q0;
    r.steps = walk_steps(pos, min(pos + min(R, n - r.q0) - 1, L - 1), a.window);
    return r;
  };
  // First token of a one-row sequence's item, and how many there are from it on.
  auto row_from = [&](int L) { return walk_start(L - 1, a.window); };

  if (tid == 0) {
    extra_row_items = 0;
    next_slot = 0;
    next_split = 0;
    next_row_slot = 0;
    next_row_split = 0;
    row_slots_needed = 0;
  }
  if (tid < 256) {
    hist[tid] = 0;
    row_hist[tid] = 0;
  }
  const PlanScan found = load_chunk(0);   // its barriers also publish the zeros above
  // tiles (of all kv heads) that run at once, one workgroup per CU
  const int lanes = max(1, kNumCUs / a.num_kv_heads);
  int chunk_tiles = kResident ? min(found.total, kPlanThreads) : found.total;
  int all_tiles = chunk_tiles, all_rows = found.set_total;
  PlanTile own = {0, 0, 0};
  // Whole tiles and one-row sequences that all run at once, in any order.
  const bool one_round = kResident && chunk_tiles + all_rows <= min(lanes, a.max_items);
  auto write_whole = [&] {
    if (tid < chunk_tiles)
      a.items[tid] = {own.idx, own.q0, 0, own.steps, -1, seq_cu[own.idx], seq_n[own.idx],
                      seq_L[own.idx]};
    if (a.rows && tid < a.num_seqs && seq_n[tid] == 1)
      a.items[chunk_tiles + found.set_before] = {tid, -1, row_from(seq_L[tid]), seq_L[tid], -1,
                                                 seq_cu[tid], 1, seq_L[tid]};
    if (tid == 0) *a.head = {chunk_tiles + all_rows, 0, 0, 0};
  };
  if constexpr (kResident) {
    if (tid < chunk_tiles) own = tile_of(tid);
    steps[tid] = own.steps;
    if (one_round && a.max_slots == 0 && a.max_row_slots == 0) {
      write_whole();
      return;
    }
  }
  // Runs tile(base, t) over every tile, dealt to the threads in turn, and
  // row(sequence, cu0, L) over every one-row sequence.
  auto each = [&](auto tile, auto row) {
    if constexpr (kResident) {
      if (tid < chunk_tiles) tile(0, own);
      if (a.rows && tid < a.num_seqs && seq_n[tid] == 1) row(tid, seq_cu[tid], seq_L[tid]);
    } else {
      all_tiles = all_rows = 0;
      for (int base = 0; base < a.num_seqs; base += kPlanThreads) {
        const PlanScan chunk = load_chunk(base);
        chunk_tiles = chunk.total;
        all_tiles += chunk_tiles;
        all_rows += chunk.set_total;
        for (int t = tid; t < chunk_tiles; t += kPlanThreads) tile(base, tile_of(t));
        if (a.rows && base + tid < a.num_seqs && seq_n[tid] == 1)
          row(base + tid, seq_cu[tid], seq_L[tid]);
        __syncthreads();
      }
    }
  };

  // ---- totals ----
  PlanTotals sum = {0.f, 0.f, 1.f, 1.f};
  each(
      [&](int, const PlanTile& t) {
        sum.steps += t.steps;
        sum.max_steps = fmaxf(sum.max_steps, t.steps);
      },
      [&](int, int, int L) {
        const int tokens = L - row_from(L);
        sum.tokens += tokens;
        sum.max_tokens = fmaxf(sum.max_tokens, tokens);
      });
  sum = plan_totals(sum, totals_lds);
  const int tiles = all_tiles, rows = all_rows;
  const int longest = (int)sum.max_steps, max_tokens = (int)fminf(sum.max_tokens, 1e9f);
  const float steps_sum = sum.steps, tokens_sum = sum.tokens;
  constexpr int kWhole = 0x7fffffff;

  // ---- one-row sequences: at least two items per CU, whole above that ----
  int row_c = kWhole, row_items = rows;
  if (rows > 0 && a.max_row_slots > 0)
    row_c = max(kRowTokens, ((int)fminf(tokens_sum / (2 * lanes), 1e9f) / 512 + 1) * 512);
  const bool share = kResident && a.max_slots > 0 &&
                     sharing_pays(longest, (long long)tiles * a.num_kv_heads, kPlanSteps);
  if constexpr (kResident) {
    if (one_round && !share && max_tokens <= row_c) {
      write_whole();
      return;
    }
  }
  if (max_tokens > row_c) {
    each([](int, const PlanTile&) {},
         [&](int, int, int L) {
           const int p = row_pieces(L - row_from(L), row_c).y;
           if (p > 1) {
             atomicAdd(&row_slots_needed, p);
             atomicAdd(&extra_row_items, p - 1);
           }
         });
    __syncthreads();
    if (row_slots_needed > a.max_row_slots) row_c = kWhole;
    else row_items += extra_row_items;
  }
  const float row_steps = tokens_sum / 64.f;
  const float row_work = kRowStep * row_steps + (float)kItemSteps * row_items;
  const float row_hbm = kRowHbmStep * a.num_kv_heads * row_steps;

  // ---- how many steps an item gets, and how tiles and one-row items mix ----
  // Candidate k limits an item to 1 / (k + 1) of the longest tile. Its time is
  // estimated as r rounds of its items on the fewest CUs that do them in r
  // rounds, while the one-row items run on the others as far as those and HBM
  // allow, and the rest of them after; without one-row items r is as few as
  // fit. The fewest items within 3% of the best win.
  PlanChoice pick = {kWhole, 1, 0, 1.f, 1.f};   // whole tiles, nothing to mix
  if (share || rows) {
    constexpr int kPer = kPlanThreads / kPlanCandidates;   // 32 lanes per candidate
    auto limit = [&](int k) { return k ? max(4, ((longest + k) / (k + 1) + 1) & ~1) : kWhole; };
    if (share) {
      const int cand = tid / kPer, mine = limit(cand);
      int items = 0, slots = 0;
      for (int t = tid % kPer; t < tiles; t += kPer) {
        const int p = tile_pieces(steps[t], mine).y;
        items += p;
        slots += p > 1 ? p : 0;
      }
#pragma unroll
      for (int o = kPer / 2; o > 0; o >>= 1) {
        items += __shfl_xor(items, o, kPer);
        slots += __shfl_xor(slots, o, kPer);
      }
      if (tid % kPer == 0) { cand_items[cand] = items; cand_slots[cand] = slots; }
    } else if (tid < kPlanCandidates) {
      cand_items[tid] = tid ? 0 : tiles;
      cand_slots[tid] = 0;
    }
    __syncthreads();
    if (tid < kPlanCandidates) {
      const int n = cand_items[tid], k = cand_slots[tid];
      PlanChoice mine = {kWhole, 1, 0, 1.f, 1.f};
      float est = INFINITY;
      if (n > 0 && k <= a.max_slots) {
        const float work = steps_sum + (float)kItemSteps * n + (float)kPartialSteps * k;
        const float each = work / n;
        const int r0 = (n + lanes - 1) / lanes;
        for (int r = r0; r < r0 + (rows ? 4 : 1); ++r) {
          const int x = (n + r - 1) / r, y = lanes - x;
          const float span = r * each;
          const float done = rows ? fminf(fminf(1.f, y * span / row_work), span / row_hbm) : 1.f;
          const float e = fmaxf(span, (work + row_work) / lanes) +
                          (1.f - done) * fmaxf(row_hbm, row_work / lanes);
          if (e < est) {
            est = e;
            mine = {limit(tid), x, y, each, rows ? y * span / fmaxf(done * row_items, 1e-3f) : 1.f};
          }
        }
      }
      float best = est;
#pragma unroll
      for (int o = kPlanCandidates / 2; o > 0; o >>= 1)
        best = fminf(best, __shfl_xor(best, o, kPlanCandidates));
      const unsigned long long good = __ballot(est <= 1.03f * best);
      if (tid == __ffsll(good) - 1) choice = mine;
    }
    __syncthreads();
    pick = choice;
    if constexpr (kResident) {
      if (one_round && !rows && pick.limit == kWhole) {
        write_whole();
        return;
      }
    }
  }
  const int C = pick.limit;
  const float per_bucket = 255.f / max(1, min(longest, C));   // C bounds an item's steps
  const float row_per_bucket = 255.f / max(1, min(max_tokens, row_c));

  // ---- items in descending length, so that the last to start are short ----
  auto bucket = [&](int per) { return 255 - min(255, (int)(per * per_bucket)); };
  auto row_bucket = [&](int per) { return 255 - min(255, (int)(per * row_per_bucket)); };
  each(
      [&](int, const PlanTile& t) {
        const int2 p = tile_pieces(t.steps, C);
        atomicAdd(&hist[bucket(p.x)], p.y);
      },
      [&](int, int, int L) {
        const int2 p = row_pieces(L - row_from(L), row_c);
        atomicAdd(&row_hist[row_bucket(p.x)], p.y);
      });
  __syncthreads();
  const PlanScan at = plan_scan(tid < 256 ? hist[tid] : 0, false, scan_lds);
  const int total = at.total;
  int row_total = 0;
  if (rows) {
    const PlanScan row_at = plan_scan(tid < 256 ? row_hist[tid] : 0, false, scan_lds);
    row_total = row_at.total;
    if (tid < 256) row_hist[tid] = row_at.before;
  }
  if (tid < 256) hist[tid] = at.before;
  __syncthreads();
  // ---- one list in the order of planned starts ----
  // Tile item j starts at (j / x) dt, one-row item k at (k / y) dd (times in
  // 1/16 steps); on a tie the tile is first. y 0: one-row items after all tiles.
  const int x = max(1, pick.x), y = pick.y;
  const long long dt = max(1, (int)(pick.tile_time * 16.f));
  const long long dd = max(1, (int)fminf(pick.row_time * 16.f, 1e9f));
  auto tile_pos = [&](int j) {
    if (row_total == 0 || y <= 0) return j;
    const long long before = ((j / x) * dt + dd - 1) / dd * y;
    return j + (int)min(before, (long long)row_total);
  };
  auto row_pos = [&](int k) {
    if (y <= 0) return total + k;
    const long long before = ((k / y) * dd / dt + 1) * x;
    return k + (int)min(before, (long long)total);
  };
  each(
      [&](int base, const PlanTile& t) {
        const int2 p = tile_pieces(t.steps, C);
        const int j0 = atomicAdd(&hist[bucket(p.x)], p.y);
        const int cu0 = seq_cu[t.idx], n = seq_n[t.idx], L = seq_L[t.idx];
        int slot = -1;
        if (p.y > 1) {
          slot = atomicAdd(&next_slot, p.y);
          const int k = atomicAdd(&next_split, 1);
          a.splits[k] = {cu0 + t.q0, min(R, n - t.q0), slot, p.y};
        }
        for (int k = 0; k < p.y; ++k) {
          const int pos = tile_pos(j0 + k);
          if (pos < a.max_items)
            a.items[pos] = {base + t.idx, t.q0, k * p.x, min(t.steps, (k + 1) * p.x),
                            slot < 0 ? -1 : slot + k, cu0, n, L};
        }
      },
      [&](int s, int cu0, int L) {
        const int from = row_from(L);
        const int2 p = row_pieces(L - from, row_c);
        const int k0 = atomicAdd(&row_hist[row_bucket(p.x)], p.y);
        int slot = -1;
        if (p.y > 1) {
          slot = atomicAdd(&next_row_slot, p.y);
          const int k = atomicAdd(&next_row_split, 1);
          a.row_splits[k] = {cu0, slot, p.y, 0};
        }
        for (int k = 0; k < p.y; ++k) {
          const int pos = row_pos(k0 + k);
          if (pos < a.max_items)
            a.items[pos] = {s, -1, from + k * p.x, min(L, from + (k + 1) * p.x),
                            slot < 0 ? -1 : slot + k, cu0, 1, L};
        }
      });
  __syncthreads();
  if (tid == 0)
    *a.head = {min(total + row_total, a.max_items), next_split, next_row_split, 0};
}

// Merge the partials of the shared tiles: one workgroup per (tile, kv head,
// wavefront of the tile's 8, quarter of the dims), 32 rows of one query head.
// Bound by the latency of reading the partials, 4 KiB each: every load is a
// row's 8 bytes per lane, contiguous over the rows, and four partials' loads are
// issued together; the merged rows go through LDS to be written in 64-byte
// pieces. 7 us for 28 tiles' heads of 8 partials (26 MB); one workgroup per 32
// rows of all dims, a partial at a time, took 8.5.
template <int G>
__global__ __launch_bounds__(256) void prefill_combine_kernel(
    const PrefillPlan* __restrict__ head, const PrefillSplit* __restrict__ splits,
    const RowSplit* __restrict__ row_splits, const uint8_t* __restrict__ slots,
    const uint8_t* __restrict__ row_slots, uint16_t* __restrict__ out, int num_q_heads,
    int num_kv_heads) {
  constexpr int kPart = kCombineParts;
  __shared__ uint32_t tile[32][kD / 2 / kPart + 1];
  const int row_tasks = head->row_splits * num_kv_heads;
  for (int task = gridDim.x - 1 - blockIdx.x; task < row_tasks; task += gridDim.x) {
    const RowSplit sp = row_splits[task / num_kv_heads];
    const int g = task % num_kv_heads;
    const size_t stride = (size_t)num_kv_heads * row_slot_bytes(G);
    const uint8_t* base = row_slots + ((size_t)sp.slot0 * num_kv_heads + g) * row_slot_bytes(G);
    for (int e = threadIdx.x; e < G * kD; e += 256) {
      merge_states<float>(
          sp.pieces, [&](int j) { return reinterpret_cast<const float*>(base + j * stride)[e]; },
          [&](int j) {
            return reinterpret_cast<const float2*>(base + j * stride +
                                                   G * kD * sizeof(float))[e / kD];
          },
          [&](float, float l, float o) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            out[((size_t)sp.row * num_q_heads + g * G) * kD + e] = to_bf16(o * inv);
          });
    }
  }
  const int tasks = head->splits * num_kv_heads * kWaves * kPart;   // of shared tiles
  for (int task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int part = task % kPart;
    const int w = (task / kPart) % kWaves;
    const int g = (task / (kPart * kWaves)) % num_kv_heads;
    const PrefillSplit sp = splits[task / (kPart * kWaves * num_kv_heads)];
    const int r0 = (w / G) * 32;
    if (r0 >= sp.rows) continue;
    constexpr int kDimPairs = kD / 2 / kPart;          // of this workgroup
    constexpr int kPer = kDimPairs / 8;                // of a thread: p0 + 8 i
    constexpr int kBatch = 4;
    const int row = threadIdx.x % 32, p0 = threadIdx.x / 32;
    const size_t stride = (size_t)num_kv_heads * kSlotBytes;
    const uint8_t* base = slots + ((size_t)sp.slot0 * num_kv_heads + g) * kSlotBytes;
    const uint8_t* ml_base = base + (size_t)kSlotFloats * sizeof(float) +
                             (w * 32 + row) * sizeof(float2);
    const uint8_t* o_base = base + ((w * (kD / 2) + part * kDimPairs + p0) * 32 + row) *
                                       sizeof(float2);

    float m = -INFINITY, l = 0.f;
    float2 o[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = make_float2(0.f, 0.f);
    for (int j0 = 0; j0 < sp.pieces; j0 += kBatch) {
      float2 ml[kBatch], v[kBatch][kPer];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {   // past the end: the last partial, at weight 0
        const size_t at = (size_t)min(j0 + b, sp.pieces - 1) * stride;
        ml[b] = *reinterpret_cast<const float2*>(ml_base + at);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          v[b][i] = *reinterpret_cast<const float2*>(o_base + at + i * 8 * 32 * sizeof(float2));
      }
      float mn = m;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) mn = fmaxf(mn, ml[b].x);
      const float ref = (mn == -INFINITY) ? 0.f : mn;
      const float alpha = fast_exp2(m - ref);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < kPer; ++i) { o[i].x *= alpha; o[i].y *= alpha; }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (j0 + b >= sp.pieces) break;
        const float wgt = fast_exp2(ml[b].x - ref);
        l = fmaf(wgt, ml[b].y, l);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          o[i].x = fmaf(wgt, v[b][i].x, o[i].x);
          o[i].y = fmaf(wgt, v[b][i].y, o[i].y);
        }
      }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      tile[row][p0 + 8 * i] = pack_bf16x2(o[i].x * inv, o[i].y * inv);
    __syncthreads();
    const int nrows = min(32, sp.rows - r0);
    const int h = g * G + w % G;
    for (int e = threadIdx.x; e < nrows * kDimPairs; e += 256) {
      const int r = e / kDimPairs, d2 = e % kDimPairs;
      reinterpret_cast<uint32_t*>(out)[((size_t)(sp.row0 + r0 + r) * num_q_heads + h) * (kD / 2) +
                                       part * kDimPairs + d2] = tile[r][d2];
    }
    __syncthreads();   // the next task writes the tile
  }
}

// Work tiles only: one workgroup per (item or tile, kv head).
template <int G, bool kPow2Blocks>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads),
                          amdgpu_waves_per_eu(2, 2)))
void prefill_kernel(const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
                    int num_blocks, const int* __restrict__ block_table,
                    const int* __restrict__ seq_lens, const int* __restrict__ cu,
                    uint16_t* __restrict__ out, const int2* __restrict__ tiles,
                    const int* __restrict__ tile_count, const PrefillItem* __restrict__ items,
                    uint8_t* __restrict__ slots, int total_q, int num_q_heads, int num_kv_heads,
                    int max_blocks, int max_seq_len, float scale_log2) {
  constexpr int kRows = 32 * kWaves / G;   // rows per work tile
  const int g = blockIdx.x % num_kv_heads;
  const int ti = blockIdx.x / num_kv_heads;
  PrefillItem it;
  if (items) it = items[ti];   // the list has room for the whole grid: read beside the count
  if (ti >= *tile_count) return;
  if (!items)   // no plan: the tile map's whole tiles
    it = whole_tile(tiles, ti, cu, seq_lens, total_q, kRows, min(max_seq_len, max_blocks * kBS),
                    kNoWindow);
  prefill_tile<G, kPow2Blocks>(it, g, q, kv, num_blocks, block_table, out, slots, num_q_heads,
                               num_kv_heads, max_blocks, PlainScore{scale_log2});
}

// A planned step that may hold one-row sequences.
template <int G, bool kPow2Blocks>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads),
                          amdgpu_waves_per_eu(2, 2)))
void prefill_step_kernel(const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
                         int num_blocks, const int* __restrict__ block_table,
                         uint16_t* __restrict__ out, const PrefillPlan* __restrict__ head,
                         const PrefillItem* __restrict__ items, uint8_t* __restrict__ slots,
                         uint8_t* __restrict__ row_slots, int num_q_heads, int num_kv_heads,
                         int max_blocks, float scale_log2) {
  const int g = blockIdx.x % num_kv_heads;
  const int ti = blockIdx.x / num_kv_heads;
  const PrefillItem it = items[ti];   // the list has room for the whole grid
  if (ti >= head->items) return;
  if (it.q0 < 0)
    prefill_row<G>(it, g, q, kv, num_blocks, block_table, out, row_slots, num_q_heads,
                   num_kv_heads, max_blocks, PlainScore{scale_log2});
  else
    prefill_tile<G, kPow2Blocks>(it, g, q, kv, num_blocks, block_table, out, slots, num_q_heads,
                                 num_kv_heads, max_blocks, PlainScore{scale_log2});
}

// Offsets of a planned step's pieces of the workspace.
namespace {
struct PrefillWs {
  int max_items, max_slots, max_row_slots;   // items; slots per kv head
  size_t items, splits, row_splits, slots, row_slots;   // byte offsets; the head is at 0
  size_t total;
};

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// Workgroups' worth of partial slots: the plan fills the chip once or twice.
constexpr int kSlotWorkgroups = 2 * kNumCUs;

PrefillWs prefill_ws(int num_seqs, int total_q, int group, int num_kv_heads) {
  PrefillWs w;
  const int lanes = num_kv_heads < kNumCUs ? kNumCUs / num_kv_heads : 1;
  w.max_slots = num_kv_heads <= kNumCUs ? kSlotWorkgroups / num_kv_heads : 0;
  // shared one-row sequences of T tokens in all have at most 2 T / (T / (2 lanes)) items
  w.max_row_slots = 4 * lanes + 8;
  w.max_items = total_q / (32 * kWaves / group) + num_seqs + w.max_slots + w.max_row_slots;
  w.items = 256;
  w.splits = w.items + up256((size_t)w.max_items * sizeof(PrefillItem));
  w.row_splits = w.splits + up256((size_t)(w.max_slots / 2 + 1) * sizeof(PrefillSplit));
  w.slots = w.row_splits + up256((size_t)(w.max_row_slots / 2 + 1) * sizeof(RowSplit));
  w.row_slots = w.slots + (size_t)w.max_slots * num_kv_heads * kSlotBytes;
  w.total = w.row_slots + (size_t)w.max_row_slots * num_kv_heads * row_slot_bytes(group);
  return w;
}
}  // namespace

size_t prefill_planned_bytes(int num_seqs, int total_q, int num_q_heads) {
  // the most of every group size's layout
  size_t most = 0;
  for (int group = 1; group <= 8; group *= 2) {
    if (num_q_heads % group) continue;
    const size_t t = prefill_ws(num_seqs, total_q, group, num_q_heads / group).total;
    most = t > most ? t : most;
  }
  return most;
}

template <int G>
static hipError_t launch_prefill_t(const PrefillArgs& a) {
  constexpr int kRowsPerTile = 32 * kWaves / G;
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  const PrefillWs w = prefill_ws(a.num_seqs, a.total_q_tokens, G, a.num_kv_heads);
  // Sharing tiles is weighed here by the bounds the host knows, and by the plan,
  // with room for the partials, by the lengths it finds. One sequence whose tiles
  // are not shared needs no plan: the tile map lists its tiles in the same order
  // without the passes that order several. The plan of more than kPlanThreads
  // sequences or tiles shares none.
  const long long bound = (long long)a.total_q_tokens / kRowsPerTile + a.num_seqs;
  const bool resident = a.num_seqs <= kPlanThreads && bound <= kPlanThreads;
  // what a tile and a one-row sequence walk at most
  const int window = a.mods ? window_keys(*a.mods) : kNoWindow;
  const int most_keys = std::min(a.max_seq_len, window + kRowsPerTile + kBS);
  const int most_row = std::min(a.max_seq_len, window + kBS);
  const long long steps = ((long long)most_keys + kKeys - 1) / kKeys;
  const long long tile_wgs = (long long)(a.total_q_tokens / kRowsPerTile) * a.num_kv_heads;
  const bool share = resident && sharing_pays(steps, tile_wgs, kLaunchSteps);
  // Several sequences may hold one-row ones (only the device knows), one does if
  // it is one row; with one longer sequence the kernel without that branch runs.
  const bool rows = a.num_seqs > 1 || a.total_q_tokens == 1;
  const bool planned = a.workspace_bytes >= w.total && (rows || share);
  const int2* tiles = nullptr;
  const int* count;
  const PrefillItem* items = nullptr;
  int grid_items, max_slots = 0, max_row_slots = 0;
  hipError_t e;
  if (planned) {
    max_slots = share ? w.max_slots : 0;
    PlanArgs p;
    p.cu = a.cu_seqlens_q;
    p.seq_lens = a.seq_lens;
    p.num_seqs = a.num_seqs;
    p.total_q = a.total_q_tokens;
    p.rows_per_tile = kRowsPerTile;
    p.num_kv_heads = a.num_kv_heads;
    p.max_seq_tokens = a.max_seq_len < a.max_blocks * kBS ? a.max_seq_len : a.max_blocks * kBS;
    // One-row sequences are shared from 1024 tokens on (a CU's walk of 4 us), from
    // 2048 where only they would need the merge's launch (about 4 us), or from
    // 8192 beside four or more rounds of tiles, which such a walk can hide in.
    const int shared_from = share ? kRowTokens
                            : tile_wgs < 4 * kNumCUs ? 2 * kRowTokens : 8 * kRowTokens;
    max_row_slots = rows && most_row > shared_from ? w.max_row_slots : 0;
    grid_items = (int)(bound + max_slots + max_row_slots);
    p.max_items = grid_items;
    p.max_slots = max_slots;
    p.rows = rows;
    p.max_row_slots = max_row_slots;
    p.window = window;
    p.items = reinterpret_cast<PrefillItem*>(ws + w.items);
    p.splits = reinterpret_cast<PrefillSplit*>(ws + w.splits);
    p.row_splits = reinterpret_cast<RowSplit*>(ws + w.row_splits);
    p.head = reinterpret_cast<PrefillPlan*>(ws);
    items = p.items;
    count = &p.head->items;
    trace_before(a.stream, "prefill_plan");
    hipLaunchKernelGGL(resident ? prefill_plan_kernel<true> : prefill_plan_kernel<false>, dim3(1),
                       dim3(kPlanThreads), 0, a.stream, p);
  } else {
    // One sequence of whole tiles, or a workspace of the tile list's size alone.
    int* c = reinterpret_cast<int*>(ws);
    int2* t = reinterpret_cast<int2*>(ws + 16);
    const long long max_tiles = (long long)((a.workspace_bytes - 16) / sizeof(int2));
    grid_items = (int)(bound < max_tiles ? bound : max_tiles);
    tiles = t;
    count = c;
    trace_before(a.stream, "prefill_tile_map");
    hipLaunchKernelGGL(prefill_tile_map_kernel, dim3(1), dim3(256), 0, a.stream, a.cu_seqlens_q,
                       a.num_seqs, a.total_q_tokens, kRowsPerTile, t, c, grid_items);
  }
  trace_after(a.stream);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long blocks = (long long)grid_items * a.num_kv_heads;
  if (blocks <= 0) return hipSuccess;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  trace_before(a.stream, a.mods ? (a.fp8 ? "prefill_scored_fp8" : "prefill_scored")
                         : a.fp8 ? "prefill_fp8" : "prefill");
  const unsigned kvh = (unsigned)a.num_kv_heads;
  const bool pow2 = (kvh & (kvh - 1)) == 0;
  const uint16_t* q = static_cast<const uint16_t*>(a.q);
  const uint8_t* kv = static_cast<const uint8_t*>(a.kv);
  uint16_t* out = static_cast<uint16_t*>(a.out);
  const PrefillPlan* head = reinterpret_cast<const PrefillPlan*>(ws);
  const float scale_log2 = a.scale * kLog2e;
  if (a.fp8 || a.mods) {
    const PrefillLaunch l = {(unsigned)blocks, planned ? head : nullptr, items, tiles, count,
                             ws + w.slots, ws + w.row_slots};
    e = !a.mods ? launch_prefill_fp8(a, l)
        : a.fp8 ? launch_prefill_scored_fp8(a, l) : launch_prefill_scored(a, l);
  } else if (planned && rows) {
    auto kernel = pow2 ? prefill_step_kernel<G, true> : prefill_step_kernel<G, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, a.stream, q, kv,
                       a.num_blocks, a.block_table, out, head, items, ws + w.slots,
                       ws + w.row_slots, a.num_q_heads, a.num_kv_heads, a.max_blocks,
                       scale_log2);
  } else {
    auto kernel = pow2 ? prefill_kernel<G, true> : prefill_kernel<G, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, a.stream, q, kv,
                       a.num_blocks, a.block_table, a.seq_lens, a.cu_seqlens_q, out, tiles, count,
                       items, ws + w.slots, a.total_q_tokens, a.num_q_heads, a.num_kv_heads,
                       a.max_blocks, a.max_seq_len, scale_log2);
  }
  trace_after(a.stream);
  const hipError_t last = hipGetLastError();
  if (e == hipSuccess) e = last;
  if (e != hipSuccess || (max_slots == 0 && max_row_slots == 0)) return e;
  trace_before(a.stream, "prefill_combine");
  hipLaunchKernelGGL((prefill_combine_kernel<G>), dim3(kCombineGrid), dim3(256), 0, a.stream, head,
                     reinterpret_cast<const PrefillSplit*>(ws + w.splits),
                     reinterpret_cast<const RowSplit*>(ws + w.row_splits), ws + w.slots,
                     ws + w.row_slots, out, a.num_q_heads, a.num_kv_heads);
  trace_after(a.stream);
  return hipGetLastError();
}

hipError_t launch_prefill(const PrefillArgs& a) {
  if (a.head_dim != kD) return hipErrorNotSupported;
  switch (a.num_q_heads / a.num_kv_heads) {
    case 1: return launch_prefill_t<1>(a);
    case 2: return launch_prefill_t<2>(a);
    case 4: return launch_prefill_t<4>(a);
    case 8: return launch_prefill_t<8>(a);
    default: return hipErrorNotSupported;
  }
}

}  // namespace kvattn
