// The work of a chunked-prefill tile, and of a one-row sequence, over a bf16 cache.
//
// Work tile = (kv head g, 32 * 8 / G consecutive new rows of one sequence),
// G = 1, 2, 4 or 8 query heads per kv head.
// A workgroup of 8 wavefronts (two per SIMD) owns one tile: wave w serves
// query head g * G + w % G over 32 rows. K/V steps of 64 keys (4 blocks) are
// gathered through the block table straight into LDS (global_load_lds) once
// per workgroup and shared by the G query heads of the group; three LDS
// buffers each let K be gathered three steps and V one step ahead of their
// use, with one barrier per step.
//
// Per wave and step, with v_mfma_f32_32x32x16_bf16:
//   S^T[key][row] = K[key][:] . Q[row][:]   A = K rows read from the
//       chunk-major K tile, B = Q^T held in registers for the whole kernel.
//       The A rows of a 32-key tile are loaded in a permuted key order so
//       that the accumulator of each lane ends up holding 8 consecutive keys
//       of each of the two blocks for one query row;
//   softmax over keys in the log2 domain against a per-row reference (a
//       past row max): a row's 64 scores live in two lanes (l and l + 32)
//       and the row state is lane-local. The reference is only moved, and
//       O^T and the row sum rescaled, when the row's max grows past it by
//       more than 2^8, so every exponential stays below 256, which bf16 P
//       and fp32 accumulation hold. A lane's exponentials are at most its
//       partial row sum, so a step whose partial sums all stay within 2^8
//       (nearly every step after the first) needs no row max at all; the
//       others take the exact max (one exchange between the row's two
//       lanes) and recompute the step's exponentials;
//   O^T[d][row] += V^T[d][key] P^T[key][row]   A = 16-byte runs of the
//       dim-major V tile, B = the bf16 P values of 8 consecutive keys of one
//       block, already in the lane that produced them.
// Software pipeline: while a wave computes the softmax of step i on the
// vector ALU, its matrix work is p.v of step i - 1 and q.k of step i + 1, so
// both units stay busy; the second wave of the SIMD covers the LDS latency.
// V rows are stored in LDS with their two 16-byte halves swapped on every
// other group of 8 rows, so the A reads of 16 rows hit 16 distinct bank
// groups. The causal mask (bottom-right: row i at position L - n + i sees
// keys 0 .. L - n + i) is applied only on steps that reach the diagonal or
// the end of the sequence.
#pragma once

#include <type_traits>

#include "common.hpp"
#include "decode_walk.hpp"
#include "launch.hpp"
#include "prefill_items.hpp"
#include "scoring.hpp"

namespace kvattn {

namespace {

constexpr int kTileBytes = kBS * kD * 2;   // one (block, K/V, head) tile: 4 KiB
constexpr int kKBufs = 3;                  // LDS K steps (gathered three steps ahead)
constexpr int kVBufs = 3;                  // LDS V steps (gathered one step ahead)

}  // namespace

// What only a tile's end needs.
struct TileEnd {
  uint16_t* out;    // of this kv head's first query head, row 0
  uint8_t* slots;   // of this kv head, slot 0
  int slot, cu0, n, qstride, num_kv_heads, q0;
};

// One item of a work tile. With ModScore a row sees the keys of its window alone; what slots
// before the first row's window hold has no effect.
template <int G, bool kPow2Blocks, class Score>
__device__ __forceinline__ void prefill_tile(
    const PrefillItem& it, int g, const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
    int num_blocks, const int* __restrict__ block_table, uint16_t* __restrict__ out,
    uint8_t* __restrict__ slots, int num_q_heads, int num_kv_heads, int max_blocks,
    const Score& score) {
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);  // uniform per wavefront
  const int lane = tid % kWave;
  const int h = g * G + wave % G;
  const int s = it.s, q0 = it.q0, cu0 = it.cu0, n = it.n;
  const int row0 = q0 + (wave / G) * 32;        // first row of this wave
  // With ModScore keys, table entries and steps count from the block of the first key that any
  // row of the tile sees on (walk_start); lo: that key.
  int L = __builtin_amdgcn_readfirstlane(it.L), lo = 0;
  const int* bt = block_table + (size_t)s * max_blocks;
  if constexpr (Score::kOn) {
    lo = score.first_key(L - n + q0);
    const int start = __builtin_amdgcn_readfirstlane(walk_start(L - n + q0, score.window));
    bt += start / kBS;
    lo -= start;
    L -= start;
  }
  const int c = L - n;                          // cached context before the chunk
  const int i0 = it.i0, N = it.i1;              // steps of the item
  __builtin_assume(i0 >= 0 && N >= 0);
  // The key step that is walked as step i. Biased scores grow towards a row's own key, by
  // more than the softmax's reference allows in a step where the slope is steep: those are
  // walked from the last keys to the first, so that the reference, once set, holds.
  const int ends = i0 + N - 1;
  auto at_step = [&](int i) __attribute__((always_inline)) {
    return Score::form == Form::kBias || Score::form == Form::kCap ? ends - i : i;
  };
  const bool idle = row0 >= n;                  // none of the wave's 32 rows is in the chunk
  // With ModScore the loop has no scalar registers to spare: kept in LDS until the end.
  __shared__ TileEnd lds_end;
  if constexpr (Score::kOn)
    if (tid == 0)
      lds_end = {out + (size_t)g * G * kD, slots + (size_t)g * kSlotBytes, it.slot, cu0, n,
                 num_q_heads * kD, num_kv_heads, q0};
  float slope = 0.f;
  __shared__ float lds_slope[kWaves];   // with a cap, which leaves no register for it
  if constexpr (Score::kOn) {
    slope = score.slope(h);
    if (Score::form == Form::kCap && lane == 0) lds_slope[wave] = slope;
  }

  __shared__ __attribute__((aligned(16))) uint8_t lds_k[kKBufs][kStepBlocks][kTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t lds_v[kVBufs][kStepBlocks][kTileBytes];

  // (at most 2^17 tiles of 4 KiB: 32 bits hold a block's bytes)
  using Off = std::conditional_t<Score::kOn, uint32_t, size_t>;
  const Off block_bytes = 2 * (Off)num_kv_heads * kTileBytes;
  // log2 of the block size when it is a power of two (a shift replaces the
  // 64-bit multiply in every gather's address)
  const int block_shift = kPow2Blocks ? __builtin_ctzll((size_t)block_bytes) : 0;
  const Off k_off = (Off)g * kTileBytes;
  const Off v_off = (Off)(num_kv_heads + g) * kTileBytes;
  const int qstride = num_q_heads * kD;

  const int lm = lane % 32;     // MFMA row / column index of this lane
  const int lh = lane / 32;     // which 8-wide half of the 16-wide k slice
  // Key permutation of the S^T rows: A row m = 8a + 4b + e holds key
  // 16 (a / 2) + 8 b + 4 (a % 2) + e of the 32-key tile, so accumulator
  // element i of lane l is key 16 (i / 8) + 8 (l / 32) + i % 8.
  const int ka = lm / 8, kb4 = (lm / 4) % 2, ke = lm % 4;
  const int k_blk = ka / 2;                              // block within the key tile
  const int k_slot = 8 * kb4 + 4 * (ka % 2) + ke;        // slot within the block

  // ---- Q^T operand of the wave's 32 rows, loaded once into registers ----
  // Lane (lm, lh) of k-step ks holds dims ks * 16 + lh * 8 .. + 8 of row
  // row0 + lm; rows past the chunk read the chunk's last row (never written).
  bf16x8_t qr[8];
  if (!idle) {
    const int row = min(row0 + lm, n - 1);
    const uint16_t* qrow = q + (size_t)(cu0 + row) * qstride + (size_t)h * kD + lh * 8;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
      qr[ks] = *reinterpret_cast<const bf16x8_t*>(qrow + ks * 16);
  }

  f32x16_t oacc[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;
  float m_ref = -INFINITY;   // reference max of the lane's row (log2 domain)
  float l_run = 0.f;         // lane-partial row sum

  // ---- gather of K or V of one 64-key step straight into LDS (global_load_lds) ----
  // The block ids of a step are read from the table first (step_ids), in
  // SGPRs: one 16-byte scalar load when all 4 blocks lie inside the sequence,
  // single entries otherwise; a block past L or with an id outside
  // [0, num_blocks) gets id -1. The bit mask of a step (bit kb: block kb is
  // real) lets the softmax mask its keys and patch_v zero its values.
  const int nblk = (L + kBS - 1) / kBS;   // table entries the sequence uses
  struct StepIds {
    int id[kStepBlocks];
  };
  auto step_ids = [&](int step) __attribute__((always_inline)) {
    StepIds r;
    const int b0 = at_step(step) * kStepBlocks;
    if (b0 + kStepBlocks <= nblk) {
      const i32x4_t v = scalar_entries4(bt, b0);
#pragma unroll
      for (int kb = 0; kb < kStepBlocks; ++kb) r.id[kb] = v[kb];
    } else {
#pragma unroll
      for (int kb = 0; kb < kStepBlocks; ++kb)
        r.id[kb] = b0 + kb < nblk ? scalar_entry(bt, b0 + kb) : -1;
    }
    return r;
  };
  // Ids are checked against the layer only where they are used, so that
  // nothing waits for the loads where they are issued.
  auto real_id = [&](int id) __attribute__((always_inline)) {
    return (unsigned)id < (unsigned)num_blocks;
  };
  auto id_bits = [&](const StepIds& r) __attribute__((always_inline)) {
    int bits = 0;
#pragma unroll
    for (int kb = 0; kb < kStepBlocks; ++kb) bits |= real_id(r.id[kb]) ? (1 << kb) : 0;
    return bits;
  };
  // The gather itself: a half step is 4 tiles of 4 KiB (blocks 0..3); in
  // round j wavefront w fills quarter (w + 8 j) % 4 of tile (w + 8 j) / 4, a
  // contiguous 1 KiB with 16 bytes per lane. K is copied as stored; for V the
  // lane picks the global 16 bytes that belong at its swizzled LDS position
  // (row pos / 2, half pos % 2 holds global half (pos % 2) ^ ((row >> 3) & 1)).
  // A block that is not real is read from block 0 instead (the host
  // guarantees one exists) and masked afterwards.
  auto gather = [&](auto v_tag, int step, const StepIds& ids) __attribute__((always_inline)) {
    constexpr bool kV = decltype(v_tag)::value;
    // The lane id is recomputed here rather than kept live across the step.
    const int ln = lane_id_fresh();
    const uint8_t* base[2];
    uint32_t off[2], lds[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int kb = (wave + kWaves * j) / 4;     // wave-uniform
      const int quarter = (wave + kWaves * j) % 4;
      // kb is wave / 4 + 2 j: pick the id by a uniform select, not an index
      const int id = wave < 4 ? ids.id[2 * j] : ids.id[2 * j + 1];
      const size_t id0 = real_id(id) ? (size_t)(unsigned)id : 0;
      base[j] = kv + (kPow2Blocks ? id0 << block_shift : id0 * block_bytes) + (kV ? v_off : k_off);
      const unsigned pos = quarter * kWave + (unsigned)ln;   // 16-byte position in the tile
      if constexpr (kV) {
        const unsigned vrow = pos / 2;
        off[j] = vrow * 32 + (((pos % 2) ^ ((vrow >> 3) & 1)) * 16);
        lds[j] = __builtin_amdgcn_readfirstlane(
            lds_addr(&lds_v[step % kVBufs][kb][quarter * 1024]));
      } else {
        off[j] = pos * 16;
        lds[j] = __builtin_amdgcn_readfirstlane(
            lds_addr(&lds_k[step % kKBufs][kb][quarter * 1024]));
      }
    }
    dma16x2(base[0], off[0], lds[0], base[1], off[1], lds[1]);
  };
  auto load_half = [&](auto v_tag, int step) __attribute__((always_inline)) {
    const StepIds ids = step_ids(step);
    gather(v_tag, step, ids);
    return id_bits(ids);
  };
  // Zero the V slots of a landed step that must not contribute: blocks that
  // are not real, and slots at or past L (their bytes may be NaN, and a zero
  // weight times NaN is NaN). Every wavefront patches the whole step right
  // before its own p.v reads it: the writes of different wavefronts are
  // identical and idempotent, so no barrier is needed between them. Called
  // only when such slots exist.
  auto patch_v = [&](int step, int bits) __attribute__((always_inline)) {
    const int kbase = at_step(step) * kKeys;
    // recomputed here, so no lane constant of this rare path stays live
    // across the pipelined loop
    const int ln = lane_id_fresh();
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int cidx = ln + kWave * j;            // 16-byte chunk of the 4 V tiles
      const int kb = cidx / 256;
      const int pos = cidx % 256;
      const int vrow = pos / 2;
      const int half_g = (pos % 2) ^ ((vrow >> 3) & 1);
      uint4* v = reinterpret_cast<uint4*>(&lds_v[step % kVBufs][kb][pos * 16]);
      if (!((bits >> kb) & 1)) {
        *v = make_uint4(0, 0, 0, 0);
        continue;
      }
      const int key = kbase + kb * kBS + 8 * half_g;
      auto seen = [&](int t) { return t < L && (!Score::kOn || t >= lo); };
      if (key + 8 <= L && (!Score::kOn || key >= lo)) continue;
      uint4 w4 = *v;
      uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t lo16 = seen(key + 2 * k) ? 0x0000ffffu : 0u;
        const uint32_t hi16 = seen(key + 2 * k + 1) ? 0xffff0000u : 0u;
        w[k] &= (lo16 | hi16);
      }
      *v = make_uint4(w[0], w[1], w[2], w[3]);
    }
  };
  auto step_clean = [&](int step, int bits) __attribute__((always_inline)) {
    if constexpr (Score::kOn) {
      bits = __builtin_amdgcn_readfirstlane(bits);
      asm volatile("" : "+s"(bits));   // compared each time, no mask kept
    }
    return bits == 0xf && (at_step(step) + 1) * kKeys <= L &&
           (!Score::kOn || at_step(step) * kKeys >= lo);
  };

  const int wave_pos0 = c + row0;   // position of the wave's first row
  const int v_read = lm * 32 + ((lh ^ ((lm >> 3) & 1)) * 16);

  // S^T for one step: 2 key tiles x 8 k-steps of 16 dims.
  auto qk = [&](int step, f32x16_t (&sa)[2]) {
    const int buf = step % kKBufs;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) sa[kt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const bf16x8_t b = qr[ks];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int chunk = 2 * ks + lh;
        const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(
            &lds_k[buf][2 * kt + k_blk][(chunk * kBS + k_slot) * 16]);
        sa[kt] = mfma32(a, b, sa[kt]);
      }
    }
  };
  // O^T += V^T P^T for one step: one k-step per block, 4 accumulator chains.
  // Used once per tile, after the pipelined loop; the fence after each block
  // keeps the compiler from hoisting all 16 operand reads at once, which
  // would need more registers than the kernel has left.
  auto pv = [&](int step, const bf16x8_t (&pr)[4]) {
    const int buf = step % kVBufs;
#pragma unroll
    for (int kb = 0; kb < kStepBlocks; ++kb) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const bf16x8_t a =
            *reinterpret_cast<const bf16x8_t*>(&lds_v[buf][kb][dt * 32 * 32 + v_read]);
        oacc[dt] = mfma32(a, pr[kb], oacc[dt]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Causal / length / real-block mask of one step's scores, in place; run
  // only on the steps that need it.
  auto mask_scores = [&](int step, int bits, f32x16_t (&sr)[2], float to) {
    const int kbase = at_step(step) * kKeys;
    const int ln = lane_id_fresh();   // as in patch_v
    const int qpos = wave_pos0 + ln % 32;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int kpos = kbase + kt * 32 + (i / 8) * 16 + (ln / 32) * 8 + (i % 8);
        const int blk_ok = (bits >> (2 * kt + i / 8)) & 1;
        int keep = (kpos <= qpos) & (kpos < L) & blk_ok;
        if constexpr (Score::kOn) keep &= kpos > qpos - score.window;
        sr[kt][i] = keep ? sr[kt][i] : to;
        if constexpr (Score::kOn)   // a few comparisons' masks at a time
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
  };
  auto needs_mask = [&](int step, int bits) __attribute__((always_inline)) {
    return (at_step(step) * kKeys + kKeys - 1 > wave_pos0) || !step_clean(step, bits) ||
           (Score::kOn && at_step(step) * kKeys <= wave_pos0 + 31 - score.window);
  };
  // bitsm1, bits0 .. bits3: real-block masks of steps i - 1, i .. i + 3
  int bitsm1 = 0, bits0 = 0, bits1 = 0, bits2 = 0, bits3 = 0;
  // block ids of the gathers of the coming phase: K of step i + 3 and V of
  // step i + 1, read at the end of the phase before (ahead of its barrier)
  StepIds idsK, idsV;
  f32x16_t sA[2], sB[2];    // scores of even / odd steps
  bf16x8_t pA[4], pB[4];    // P of even / odd steps

  // One pipeline step i: the matrix work (p.v of step i - 1, q.k of step
  // i + 1) next to the softmax of step i, with the gathers of K of step i + 3
  // and V of step i + 1 in between. The step ends by waiting for the gathers
  // of the earlier steps only (those of this step get the whole next step to
  // land) and a barrier;
  // then O takes the rescale of step i's softmax, between the p.v of steps
  // i - 1 and i.
  //
  // The matrix and softmax work is laid out by hand in 32 issue slots: slot
  // k issues matrix instruction k (p.v for k < 16, q.k after), the LDS read
  // of the operand five slots ahead, and one exponential with its share of
  // the row sum and bf16 packing. A wavefront issues in order, so without
  // this the vector work would queue behind runs of matrix instructions
  // instead of running beside them. The gathers' branches split the slots
  // into three blocks, and the compiler gathers most exponentials of a block
  // into one run, so some slots issue their matrix instructions back to back.
  // Holding the exponentials in their slots measured slower, and so did
  // either strict order of the step's two halves (all matrix work first, or
  // all softmax first). The row max, when a step needs it, follows the slots.
  auto phase = [&](auto qk_tag, auto pv_tag, int i, f32x16_t (&s_cur)[2],
                   f32x16_t (&s_nxt)[2], const bf16x8_t (&p_prev)[4], bf16x8_t (&p_cur)[4]) __attribute__((always_inline)) {
    constexpr bool kQK = decltype(qk_tag)::value;
    constexpr bool kPV = decltype(pv_tag)::value;
    // The block ids were read before the barrier that ends the previous
    // phase: wait for them here, while no operand read of this phase is in
    // flight, so that the operand prefetch below is never drained for them
    // (scalar loads share the lgkm counter with LDS reads and return out of
    // order).
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    if (kPV && !step_clean(i - 1, bitsm1)) patch_v(i - 1, bitsm1);
    const bool do_k = i + 3 < N, do_v = i + 1 < N;
    const bool masked = needs_mask(i, bits0);
    if constexpr (Score::form == Form::kCap)   // what a row does not see chooses no formula
      if (masked) mask_scores(i, bits0, s_cur, 0.f);
    const auto how = [&]() __attribute__((always_inline)) {
      if constexpr (Score::kOn)
        return score.prepare(s_cur, at_step(i) * kKeys - wave_pos0,
                             Score::form == Form::kCap ? lds_slope[wave] : slope,
                             lane_id_fresh());
      else
        return score.scale_log2;
    }();
    // score e with a reference taken off
    auto less = [&](int e, float r) __attribute__((always_inline)) {
      if constexpr (Score::kOn)
        return how.at(s_cur[e / 16][e % 16], e, r);
      else
        return fmaf(s_cur[e / 16][e % 16], how, -r);
    };
    if (masked) mask_scores(i, bits0, s_cur, -INFINITY);

    const int vbuf = (i + kVBufs - 1) % kVBufs;   // V of step i - 1
    const int kbuf = (i + 1) % kKBufs;            // K of step i + 1
    auto has_mfma = [&](int k) __attribute__((always_inline)) { return k < 16 ? kPV : kQK; };
    auto a_frag = [&](int k) __attribute__((always_inline)) {
      if (k < 16)
        return *reinterpret_cast<const bf16x8_t*>(
            &lds_v[vbuf][k / 4][(k % 4) * 32 * 32 + v_read]);
      const int ks = (k - 16) / 2, kt = (k - 16) % 2;
      return *reinterpret_cast<const bf16x8_t*>(
          &lds_k[kbuf][2 * kt + k_blk][((2 * ks + lh) * kBS + k_slot) * 16]);
    };
    constexpr int kAhead = kQK ? 5 : 3;   // the last step keeps fewer reads in flight
    bf16x8_t fr[kAhead + 1];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (has_mfma(k)) fr[k % (kAhead + 1)] = a_frag(k);
    }
    float ref = (m_ref == -INFINITY) ? 0.f : m_ref, alpha = 1.f, psum = 0.f;
    bool rescale = false;
    float pe[32];
    uint32_t pw[16];
    f32x16_t zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero[e] = 0.f;
    // Raised issue priority while this wavefront issues its matrix slots, so
    // that the arbiter prefers its MFMAs and operand reads over the vector
    // work of the other wavefront of the SIMD (0.5-0.9% faster, same-box A/B).
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      // operand reads for slot k + kAhead
      const int kn = k + kAhead;
      if (kn < 32 && has_mfma(kn)) fr[kn % (kAhead + 1)] = a_frag(kn);
      // matrix instruction k
      if (k < 16) {
        if (kPV) oacc[k % 4] = mfma32(fr[k % (kAhead + 1)], p_prev[k / 4], oacc[k % 4]);
      } else if (kQK) {
        const int ks = (k - 16) / 2, kt = (k - 16) % 2;
        s_nxt[kt] = mfma32(fr[k % (kAhead + 1)], qr[ks], ks == 0 ? zero : s_nxt[kt]);
      }
      // softmax share of slot k: the exponential of score k against the
      // current reference
      {
        const int e = k;
        pe[e] = fast_exp2(less(e, ref));
        if (e % 2 == 1) {
          // the row sum adds the bf16 values that p.v multiplies
          pw[e / 2] = pack_bf16x2(pe[e - 1], pe[e]);
          psum = dot2_bf16(pw[e / 2], kBf16OnePair, psum);
        }
      }
      // the step's gathers, issued inside the schedule (K in slot 10, V in
      // slot 26) so that their LDS writes do not land in one burst
      if (k == 10 && do_k) {
        gather(std::false_type{}, i + 3, idsK);
        bits3 = id_bits(idsK);
      }
      if (k == 26 && do_v) gather(std::true_type{}, i + 1, idsV);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    // A row without a reference yet, or a lane whose partial row sum (which
    // bounds each of its exponentials) left 2^8: take the exact row max, move
    // the reference of the rows that outgrew theirs by more than 2^8, and
    // redo the step's exponentials against it. Rows that did not outgrow
    // theirs get the same values again.
    if (__builtin_amdgcn_ballot_w64(m_ref == -INFINITY || !(psum <= kPsumBound)) != 0) {
      // with a bias the scores less the reference, as the slots computed them, and computed
      // again here, not kept from there
      float taken = 0.f;
      if constexpr (Score::form == Form::kBias) {
        taken = ref;
        asm volatile("" : "+v"(s_cur[0]), "+v"(s_cur[1]), "+v"(taken));
#pragma unroll
        for (int e = 0; e < 32; ++e) s_cur[e / 16][e % 16] = less(e, taken);
      }
      auto finished = [&](float x, float r) __attribute__((always_inline)) {
        if constexpr (!Score::kOn) return fmaf(x, how, -r);
        else if constexpr (Score::form == Form::kBias) return x - r;
        else return fmaf(x, how.by, -r);
      };
      float mp0 = -INFINITY, mp1 = -INFINITY;
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        mp0 = max3f(mp0, s_cur[e / 16][e % 16], s_cur[e / 16][e % 16 + 1]);
        mp1 = max3f(mp1, s_cur[e / 16][e % 16 + 2], s_cur[e / 16][e % 16 + 3]);
      }
      float mx = max3f(mp0, mp1, mp1);
      mx = max3f(mx, __shfl_xor(mx, 32, kWave), mx);
      const float tmax = finished(mx, -taken);
      const bool grow = tmax > m_ref + kLazyRescale;
      rescale = __builtin_amdgcn_ballot_w64(grow) != 0;
      const float nref = grow ? tmax : m_ref;
      alpha = (m_ref == -INFINITY) ? 0.f : fast_exp2(m_ref - nref);
      m_ref = nref;
      ref = (nref == -INFINITY) ? 0.f : nref;
      psum = 0.f;
      const float more = ref - taken;
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        pw[e / 2] = pack_bf16x2(fast_exp2(finished(s_cur[e / 16][e % 16], more)),
                                fast_exp2(finished(s_cur[e / 16][e % 16 + 1], more)));
        psum = dot2_bf16(pw[e / 2], kBf16OnePair, psum);
      }
    }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
      p_cur[kb] = __builtin_bit_cast(
          bf16x8_t, make_uint4(pw[4 * kb], pw[4 * kb + 1], pw[4 * kb + 2], pw[4 * kb + 3]));
    l_run = l_run * alpha + psum;
    // keep the softmax in its slots (the compiler would otherwise sink it
    // next to its first use, away from the matrix work it should overlap)
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("" ::"v"(p_cur[k]));
    asm volatile("" ::"v"(l_run));
    // the block ids of the next phase's gathers
    if (i + 4 < N) idsK = step_ids(i + 4);
    if (i + 2 < N) idsV = step_ids(i + 2);
    // wait for the gathers of steps before this one (each thread issued two
    // for K when i + 3 < N and two for V when i + 1 < N in this step)
    if (i + 3 < N)
      asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else if (i + 1 < N)
      asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (rescale) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) oacc[dt] *= alpha;
    }
    bitsm1 = bits0;
    bits0 = bits1;
    bits1 = bits2;
    bits2 = bits3;
  };

  // A wavefront none of whose rows lies in the chunk (a short chunk's last
  // tile, a one-row decode sequence in a unified batch) still takes its share
  // of every gather and meets every barrier, step for step like the others,
  // but does no matrix or softmax work and writes nothing.
  if (idle) {
    if (N > i0) {
      load_half(std::false_type{}, i0);
      if (i0 + 1 < N) load_half(std::false_type{}, i0 + 1);
      if (i0 + 2 < N) load_half(std::false_type{}, i0 + 2);
      load_half(std::true_type{}, i0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      __syncthreads();   // the others' q.k of the first step
      for (int i = i0; i < N; ++i) {
        if (i + 3 < N) load_half(std::false_type{}, i + 3);
        if (i + 1 < N) load_half(std::true_type{}, i + 1);
        if (i + 3 < N)
          asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        else if (i + 1 < N)
          asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
        else
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
      }
    }
    return;
  }

  if (N > i0) {
    bits0 = load_half(std::false_type{}, i0);
    if (i0 + 1 < N) bits1 = load_half(std::false_type{}, i0 + 1);
    if (i0 + 2 < N) bits2 = load_half(std::false_type{}, i0 + 2);
    load_half(std::true_type{}, i0);
    if (i0 + 3 < N) idsK = step_ids(i0 + 3);
    if (i0 + 1 < N) idsV = step_ids(i0 + 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    qk(i0, sA);
    __syncthreads();   // K of the first step is read; its pipeline step gathers into its buffer
    constexpr std::true_type T{};
    constexpr std::false_type F{};
    if (i0 + 1 < N)
      phase(T, F, i0, sA, sB, pB, pA);
    else
      phase(F, F, i0, sA, sB, pB, pA);
    int i = i0 + 1;   // i0 is even: even steps use sA and pA
    for (; i + 1 <= N - 2; i += 2) {
      phase(T, T, i, sB, sA, pA, pB);
      phase(T, T, i + 1, sA, sB, pB, pA);
    }
    if (i <= N - 2) {
      phase(T, T, i, sB, sA, pA, pB);
      ++i;
    }
    // p.v of the last step (its V landed by the last step's full wait)
    int second = i0 + 1;
    if constexpr (Score::kOn)   // compared again here, not kept as a mask over the loop
      asm volatile("" : "+s"(second));
    if (second < N) {
      if (i & 1)
        phase(F, T, i, sB, sA, pA, pB);
      else
        phase(F, T, i, sA, sB, pB, pA);
    }
    if (!step_clean(N - 1, bitsm1)) patch_v(N - 1, bitsm1);
    pv(N - 1, ((N - 1) & 1) ? pB : pA);
  }

  // ---- write O (this lane: row lm): normalised, or the item's partial ----
  {
    TileEnd end;
    int wv = wave;
    if constexpr (Score::kOn) {
      int first = i0;
      asm volatile("" : "+s"(first), "+s"(wv));   // as above
      if (N <= first) __syncthreads();  // no step has published lds_end
      end = lds_end;
      end.slot = __builtin_amdgcn_readfirstlane(end.slot);
    } else {
      end = {out + (size_t)g * G * kD, slots + (size_t)g * kSlotBytes, it.slot, cu0, n, qstride,
             num_kv_heads, q0};
    }
    const int row0 = end.q0 + (wv / G) * 32;
    const float lt = l_run + __shfl_xor(l_run, 32, kWave);
    const int r = row0 + lm;
    if (end.slot < 0) {
      // A lane holds 8-byte pieces of its row, two lanes per row: stored like
      // that, an instruction touches 32 rows of 16 bytes. Half the dims at a
      // time go through the wavefront's part of the K buffers, which nobody
      // reads any more, and are stored in runs of 128 bytes. A call, stored directly and
      // like this: 7 fresh prompts of 188 to 2031 rows (64 query heads over 8)
      // 172 -> 159 us, 64 of 100 rows (32 over 8) 59 -> 51 us, 4 of 64 rows 12.8 ->
      // 10.6 us; tiles of hundreds of steps do not notice.
      constexpr int kHalf = kD / 2, kRowBytes = kHalf * 2 + 16;   // padded against conflicts
      static_assert(kWaves * 32 * kRowBytes <= (int)sizeof(lds_k), "fits the K buffers");
      uint8_t* stage = &lds_k[0][0][0] + wv * 32 * kRowBytes;
      const float inv = lt > 0.f ? 1.f / lt : 0.f;
      const int sr = lane / 16, sc = lane % 16;   // row of four, 8-byte piece of its half
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int dt = 2 * half; dt < 2 * half + 2; ++dt) {
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const f32x16_t& o = oacc[dt];
            *reinterpret_cast<uint2*>(stage + lm * kRowBytes +
                                      ((dt - 2 * half) * 32 + a * 8 + lh * 4) * 2) =
                make_uint2(pack_bf16x2(o[4 * a + 0] * inv, o[4 * a + 1] * inv),
                           pack_bf16x2(o[4 * a + 2] * inv, o[4 * a + 3] * inv));
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int rr = 4 * j + sr;
          const uint2 x = *reinterpret_cast<const uint2*>(stage + rr * kRowBytes + sc * 8);
          if (row0 + rr < end.n)
            *reinterpret_cast<uint2*>(end.out +
                                      (size_t)(end.cu0 + row0 + rr) * end.qstride +
                                      (wv % G) * kD + half * kHalf + sc * 4) = x;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    } else if (r < end.n) {
      uint8_t* slot = end.slots + (size_t)end.slot * end.num_kv_heads * kSlotBytes;
      float2* po = reinterpret_cast<float2*>(slot) + wv * 32 * (kD / 2) + lm;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int a = 0; a < 8; ++a)   // dims dt 32 + (a / 2) 8 + lh 4 + (a % 2) 2 .. + 2
          po[(dt * 16 + (a / 2) * 4 + lh * 2 + a % 2) * 32] =
              make_float2(oacc[dt][2 * a], oacc[dt][2 * a + 1]);
      if (lh == 0)
        reinterpret_cast<float2*>(slot + kSlotFloats * sizeof(float))[wv * 32 + lm] =
            make_float2(m_ref, lt);
    }
  }
}

// One item of a one-row sequence: the eight wavefronts share its tokens evenly
// in whole steps of 64 and merge their states through LDS.
template <int G, class Score>
__device__ __forceinline__ void prefill_row(
    const PrefillItem& it, int g, const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
    int num_blocks, const int* __restrict__ block_table, uint16_t* __restrict__ out,
    uint8_t* __restrict__ row_slots, int num_q_heads, int num_kv_heads, int max_blocks,
    const Score& score) {
  __shared__ __attribute__((aligned(16))) float o_lds[kWaves][G * kD];
  __shared__ float2 ml_lds[kWaves][G];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.i0, i1 = it.i1;
  const int per = max(1, (i1 - i0 + kWaves * kKeys - 1) / (kWaves * kKeys)) * kKeys;
  const int parts = (i1 - i0 + per - 1) / per;     // wavefronts with tokens
  const size_t head_off = (size_t)g * kTileBytes;
  const DecodeTiles<false> tiles = {kv, nullptr, 0, 2 * (size_t)num_kv_heads * kTileBytes,
                                    head_off, (size_t)num_kv_heads * kTileBytes + head_off};
  const size_t row = ((size_t)it.cu0 * num_q_heads + g * G) * kD;
  int lo = 0;
  if constexpr (Score::kOn) lo = score.first_key(it.L - 1);
  if (wave < parts) {
    const int t0 = i0 + wave * per;
    walk_bf16<kD, G, false, false>(tiles, q + row, block_table + (size_t)it.s * max_blocks,
                                   num_blocks, t0, min(i1, t0 + per), score, o_lds[wave],
                                   ml_lds[wave], g * G, it.L - 1, lo);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * kD; e += kThreads) {
    merge_states<float>(
        parts, [&](int j) { return o_lds[j][e]; }, [&](int j) { return ml_lds[j][e / kD]; },
        [&](float m, float l, float o) {
          if (it.slot < 0) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            out[row + e] = to_bf16(o * inv);
          } else {
            uint8_t* slot = row_slots + ((size_t)it.slot * num_kv_heads + g) * row_slot_bytes(G);
            reinterpret_cast<float*>(slot)[e] = o;
            if (e % kD == 0)
              reinterpret_cast<float2*>(slot + G * kD * sizeof(float))[e / kD] =
                  make_float2(m, l);
          }
        });
  }
}

}  // namespace kvattn
