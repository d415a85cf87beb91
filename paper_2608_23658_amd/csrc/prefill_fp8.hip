// Chunked-prefill attention over a cache in 8 bits: the tiles, plan, partials and
// merge of the bf16 prefill, with a tile pipeline that converts what it gathers.
//
// A step's K and V (64 keys) are 8 KiB each: 16 bytes a thread. Each thread loads its
// piece into registers one step ahead, converts it to bf16 times its block's power of
// two, exactly, and writes it into the LDS tiles that the products read, in the order
// the bf16 tiles have. Sixteen conversions a thread and step serve all eight
// wavefronts; converting on the way from LDS to the matrix unit instead would take
// each wavefront 128, beside a vector unit that the softmax fills. The products, the
// softmax and its lazy reference, the partials and the output are those of the bf16
// tile, and so is what bounds a step: the matrix unit, the vector unit and LDS reads
// (256 KiB for 1 MiFLOP of each of 8 wavefronts) in nearly equal parts.
//
// 8192 rows over 24576 cached tokens, 32 query heads over 8, on one box after
// another (the bf16 kernel takes 3.27 to 3.32 ms):
//   gathered into raw LDS buffers, read back, converted and written     3.88 ms
//   buffers' addresses as constants, one address for a lane's writes     0.93 of that
//   no branch among the issue slots, the last step in one form           0.88
//   through registers instead of LDS, addresses held, no raised priority 0.86
// (The branch had made the compiler sink half of a step's exponentials behind it.)
//
// Slots that must not contribute (past the sequence's end, or of a block id
// outside the layer) are zeroed in V as they are converted and masked in the scores.

#include <type_traits>

#include "common.hpp"
#include "kv_fp8.hpp"
#include "launch.hpp"
#include "prefill_items.hpp"

namespace kvattn {

namespace {
constexpr int kTile = kBS * kD * 2;      // the same in bf16
constexpr int kBufs = 2;                 // LDS steps of each kind

// Four bytes at a 4-byte aligned, wave-uniform address, by a scalar load.
__device__ __forceinline__ uint32_t scalar_word(const uint8_t* p) {
  return *(const __attribute__((address_space(4))) uint32_t*)(uintptr_t)p;
}
}  // namespace

// One item of a work tile.
template <int G>
__device__ __forceinline__ void prefill_tile_fp8(
    const PrefillItem& it, int g, const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
    int num_blocks, const int* __restrict__ block_table, uint16_t* __restrict__ out,
    uint8_t* __restrict__ slots, int num_q_heads, int num_kv_heads, int max_blocks,
    float scale_log2) {
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);  // uniform per wavefront
  const int lane = tid % kWave;
  const int h = g * G + wave % G;
  const int s = it.s, q0 = it.q0, cu0 = it.cu0, n = it.n;
  const int L = __builtin_amdgcn_readfirstlane(it.L);
  const int row0 = q0 + (wave / G) * 32;        // first row of this wave
  const int c = L - n;                          // cached context before the chunk
  const int i0 = it.i0, N = it.i1;              // steps of the item
  __builtin_assume(i0 >= 0 && N >= 0);
  const bool idle = row0 >= n;                  // none of the wave's 32 rows is in the chunk

  struct Lds {
    uint8_t v[kBufs][kStepBlocks][kTile], k[kBufs][kStepBlocks][kTile];
    uint8_t more[kWaves * 32 * 144 - kBufs * kStepBlocks * kTile];   // the rows of the end
    // what only the end needs, kept off the scalar registers of the loop
    struct {
      uint16_t* out;    // of this kv head's first query head, row 0
      uint8_t* slots;   // of this kv head, slot 0
      int slot, cu0, n, qstride, num_kv_heads;
    } end;
  };
  __shared__ __attribute__((aligned(16))) Lds lds;
  if (tid == 0)
    lds.end = {out + (size_t)g * G * kD, slots + (size_t)g * kSlotBytes, it.slot, cu0, n,
               num_q_heads * kD, num_kv_heads};

  const Fp8Tiles tiles(kv, num_kv_heads, kD, g);
  const int* bt = block_table + (size_t)s * max_blocks;
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

  // ---- gather of a step into registers ----
  // The block ids of a step are read from the table first (step_ids), in
  // SGPRs: one 16-byte scalar load when all 4 blocks lie inside the sequence,
  // single entries otherwise; a block past L or with an id outside
  // [0, num_blocks) counts as id -1 and is read from block 0 instead (the host
  // guarantees one exists). The bit mask of a step (bit kb: block kb is real) lets
  // the softmax mask its keys.
  const int nblk = (L + kBS - 1) / kBS;   // table entries the sequence uses
  struct StepIds {
    int id[kStepBlocks];
  };
  auto step_ids = [&](int step) __attribute__((always_inline)) {
    StepIds r;
    const int b0 = step * kStepBlocks;
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
  auto real_id = [&](int id) __attribute__((always_inline)) {
    return (unsigned)id < (unsigned)num_blocks;
  };
  auto id_bits = [&](const StepIds& r) __attribute__((always_inline)) {
    int bits = 0;
#pragma unroll
    for (int kb = 0; kb < kStepBlocks; ++kb) bits |= real_id(r.id[kb]) ? (1 << kb) : 0;
    return bits;
  };
  // Wavefront w gathers and converts half w % 2 (dims 64 (w % 2) .. + 64) of the
  // tiles of block w / 2 of a step.
  const int my_kb = wave / 2, my_half = wave % 2;
  // This wavefront's block of a step alone, and an id as it counts.
  auto my_entry = [&](int step) __attribute__((always_inline)) {
    const int b = step * kStepBlocks + my_kb;
    return b < nblk ? scalar_entry(bt, b) : -1;
  };
  auto real = [&](int id) __attribute__((always_inline)) { return real_id(id) ? id : -1; };
  auto my_block = [&](int id) __attribute__((always_inline)) { return tiles.block(max(id, 0)); };
  // This lane's 16 bytes of the K or V tile (at part) of a block.
  auto gather = [&](int id, uint32_t part) __attribute__((always_inline)) {
    return *reinterpret_cast<const uint4*>(my_block(id) + (part + my_half * 1024) +
                                           (uint32_t)lane * 16);
  };
  uint4 rk, rv;   // of K of step i + 2 and V of step i, at the beginning of phase i
  // The exponents of a block, K's in the low byte.
  const int e_shift = (tiles.e_off & 2) * 8;
  auto exps_of = [&](int id) __attribute__((always_inline)) {
    return scalar_word(my_block(id) + (tiles.e_off & ~3u));
  };
  auto k_scale = [&](uint32_t w) { return fp8_scale((w >> e_shift) & 0xff); };
  // In place of a block that is not there block 0 is read, with codes set to zero; its byte
  // may be 255 if nobody has written it, a scale that makes NaN of zero too: at most 254.
  auto v_scale = [&](uint32_t w) { return fp8_scale(min((w >> (e_shift + 8)) & 0xff, 254u)); };
  // Where the lane's converted pieces go. K: 16 dims of one token are two 16-byte
  // chunks of the chunk-major tile. V: dword w is tokens 4 (lane / 16) .. + 4 of dim
  // 64 half + 16 w + lane % 16, eight bytes of its row; a row's two 16-byte halves are
  // swapped on every other group of 8.
  const int k_at = my_kb * kTile + ((2 * (my_half * 4 + lane / 16)) * kBS + lane % 16) * 16;
  const int v_at = my_kb * kTile + (my_half * 64 + lane % 16) * 32 +
                   ((lane / 32) ^ ((lane >> 3) & 1)) * 16 + (lane / 16 % 2) * 8;
  auto put_k = [&](int buf, int at, int part, uint32_t a, uint32_t b,
                   float scale) __attribute__((always_inline)) {
    *reinterpret_cast<bf16x8_t*>(&lds.k[buf][0][at + part * kBS * 16]) =
        fp8x8_to_bf16(a, b, scale, scale);
  };
  auto put_v = [&](int buf, int at, int w, uint32_t a, float scale) __attribute__((always_inline)) {
    *reinterpret_cast<uint2*>(&lds.v[buf][0][at + w * 512]) = fp8x4_to_bf16(a, scale);
  };
  // Whether this wavefront's V block of a step holds slots that must not contribute.
  auto v_masked = [&](int step, int id) __attribute__((always_inline)) {
    return id < 0 || step * kKeys + (my_kb + 1) * kBS > L;
  };
  auto v_patch = [&](int step, int id) __attribute__((always_inline)) {
    const unsigned ln = lane_id_fresh();
    const uint32_t keep =
        id < 0 ? 0u : first_bytes(L - (step * kKeys + my_kb * kBS + (int)(ln / 16) * 4));
    rv = make_uint4(rv.x & keep, rv.y & keep, rv.z & keep, rv.w & keep);
  };
  auto convert_k = [&](int step, uint32_t exps) __attribute__((always_inline)) {
    const int buf = step % kBufs;
    put_k(buf, k_at, 0, rk.x, rk.y, k_scale(exps));
    put_k(buf, k_at, 1, rk.z, rk.w, k_scale(exps));
  };
  auto convert_v = [&](int step, int id, uint32_t exps) __attribute__((always_inline)) {
    const int buf = step % kBufs;
    if (v_masked(step, id)) v_patch(step, id);
    put_v(buf, v_at, 0, rv.x, v_scale(exps));
    put_v(buf, v_at, 1, rv.y, v_scale(exps));
    put_v(buf, v_at, 2, rv.z, v_scale(exps));
    put_v(buf, v_at, 3, rv.w, v_scale(exps));
  };
  auto step_clean = [&](int step, int bits) __attribute__((always_inline)) {
    return bits == 0xf && (step + 1) * kKeys <= L;
  };

  const int wave_pos0 = c + row0;   // position of the wave's first row
  const int v_read = lm * 32 + ((lh ^ ((lm >> 3) & 1)) * 16);

  // S^T for one step: 2 key tiles x 8 k-steps of 16 dims.
  auto qk = [&](int step, f32x16_t (&sa)[2]) {
    const int buf = step % kBufs;
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
            &lds.k[buf][2 * kt + k_blk][(chunk * kBS + k_slot) * 16]);
        sa[kt] = mfma32(a, b, sa[kt]);
      }
    }
  };
  // O^T += V^T P^T for one step: one k-step per block, 4 accumulator chains.
  // Used once per tile, after the pipelined loop; the fence after each block
  // keeps the compiler from hoisting all 16 operand reads at once, which
  // would need more registers than the kernel has left.
  auto pv = [&](int step, const bf16x8_t (&pr)[4]) {
    const int buf = step % kBufs;
#pragma unroll
    for (int kb = 0; kb < kStepBlocks; ++kb) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const bf16x8_t a =
            *reinterpret_cast<const bf16x8_t*>(&lds.v[buf][kb][dt * 32 * 32 + v_read]);
        oacc[dt] = mfma32(a, pr[kb], oacc[dt]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Causal / length / real-block mask of one step's scores, in place; run
  // only on the steps that need it.
  auto mask_scores = [&](int step, int bits, f32x16_t (&sr)[2]) {
    const int kbase = step * kKeys;
    const int ln = lane_id_fresh();
    const int qpos = wave_pos0 + ln % 32;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int kpos = kbase + kt * 32 + (i / 8) * 16 + (ln / 32) * 8 + (i % 8);
        const int blk_ok = (bits >> (2 * kt + i / 8)) & 1;
        const int keep = (kpos <= qpos) & (kpos < L) & blk_ok;
        sr[kt][i] = keep ? sr[kt][i] : -INFINITY;
      }
  };
  auto needs_mask = [&](int step, int bits) __attribute__((always_inline)) {
    return (step * kKeys + kKeys - 1 > wave_pos0) || !step_clean(step, bits);
  };
  // real-block masks of steps i .. i + 3, four bits each
  int bits = 0;
  // block ids of the gathers of the coming phase: K of step i + 3 and this
  // wavefront's of V of step i + 1, read at the end of the phase before (ahead of its barrier)
  StepIds idsK = {{-1, -1, -1, -1}};
  int idK = -1, idV = -1;
  // of what the coming phase converts (rk, rv), K of step i + 2 and V of step
  // i: this wavefront's V block, and the words that hold their exponents
  int v_id = -1;
  uint32_t k_exps = 0, v_exps = 0;
  f32x16_t sA[2], sB[2];    // scores of even / odd steps
  bf16x8_t pA[4], pB[4];    // P of even / odd steps

  // One pipeline step i: the matrix work (p.v of step i - 1, q.k of step
  // i + 1) next to the softmax of step i, the conversion of K of step i + 2 and V
  // of step i, gathered in the phase before, and the gathers of K of step
  // i + 3 and V of step i + 1. The step ends with a barrier; then O takes the
  // rescale of step i's softmax, between the p.v of steps i - 1 and i.
  //
  // As in the bf16 tile, the work is laid out by hand in 32 issue slots: slot k
  // issues matrix instruction k (p.v for k < 16, q.k after), the LDS read of the
  // operand five slots ahead, one exponential with its share of the row sum and
  // bf16 packing, and some a part of the conversion. The slots are one block without a
  // branch, so the exponentials stay in theirs. The row max, when a step needs it,
  // follows them.
  // parity: i % 2, in the loop a constant, so that the buffers' addresses are too.
  auto phase = [&](auto qk_tag, auto pv_tag, auto parity, int i, f32x16_t (&s_cur)[2],
                   f32x16_t (&s_nxt)[2], const bf16x8_t (&p_prev)[4],
                   bf16x8_t (&p_cur)[4]) __attribute__((always_inline)) {
    constexpr bool kQK = decltype(qk_tag)::value;
    constexpr bool kPV = decltype(pv_tag)::value;
    const int cur = parity, nxt = 1 - cur;   // buffers of steps i and i + 1
    // The block ids were read before the barrier that ends the previous
    // phase: wait for them here, while no operand read of this phase is in
    // flight, so that the operand prefetch below is never drained for them
    // (scalar loads share the lgkm counter with LDS reads and return out of
    // order).
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    if (needs_mask(i, bits & 0xf)) mask_scores(i, bits & 0xf, s_cur);
    // here and not where it is converted, so that no branch splits the slots
    if (v_masked(i, v_id)) v_patch(i, v_id);

    const int vbuf = nxt;   // V of step i - 1
    const int kbuf = nxt;   // K of step i + 1
    auto has_mfma = [&](int k) __attribute__((always_inline)) { return k < 16 ? kPV : kQK; };
    auto a_frag = [&](int k) __attribute__((always_inline)) {
      if (k < 16)
        return *reinterpret_cast<const bf16x8_t*>(
            &lds.v[vbuf][k / 4][(k % 4) * 32 * 32 + v_read]);
      const int ks = (k - 16) / 2, kt = (k - 16) % 2;
      return *reinterpret_cast<const bf16x8_t*>(
          &lds.k[kbuf][2 * kt + k_blk][((2 * ks + lh) * kBS + k_slot) * 16]);
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
    constexpr int kConvSlot = 6;
    const int new_k = kQK ? real(idK) : -1, new_v = kQK ? real(idV) : -1;
    if (kQK) bits |= id_bits(idsK) << 12;
    f32x16_t zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero[e] = 0.f;
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
        pe[e] = fast_exp2(fmaf(s_cur[e / 16][e % 16], scale_log2, -ref));
        if (e % 2 == 1) {
          // A weight is rounded to bf16, as the matrix instruction takes it (at most 2^-8
          // of it); the row sum adds the rounded ones, so that they add up to one.
          pw[e / 2] = pack_bf16x2(pe[e - 1], pe[e]);
          psum = dot2_bf16(pw[e / 2], kBf16OnePair, psum);
        }
      }
      if (k == kConvSlot + 1 && kQK) put_k(cur, k_at, 0, rk.x, rk.y, k_scale(k_exps));
      if (k == kConvSlot + 3 && kQK) put_k(cur, k_at, 1, rk.z, rk.w, k_scale(k_exps));
      if (k == kConvSlot + 4 && kQK) rk = gather(new_k, tiles.k_off);
      if (k == kConvSlot + 6) put_v(cur, v_at, 0, rv.x, v_scale(v_exps));
      if (k == kConvSlot + 8) put_v(cur, v_at, 1, rv.y, v_scale(v_exps));
      if (k == kConvSlot + 10) put_v(cur, v_at, 2, rv.z, v_scale(v_exps));
      if (k == kConvSlot + 12) put_v(cur, v_at, 3, rv.w, v_scale(v_exps));
      if (k == kConvSlot + 13 && kQK) rv = gather(new_v, tiles.v_off);
      __builtin_amdgcn_sched_barrier(0);
    }
    // A row without a reference yet, or a lane whose partial row sum (which
    // bounds each of its exponentials) left 2^8: take the exact row max, move
    // the reference of the rows that outgrew theirs by more than 2^8, and
    // redo the step's exponentials against it. Rows that did not outgrow
    // theirs get the same values again.
    if (__builtin_amdgcn_ballot_w64(m_ref == -INFINITY || !(psum <= kPsumBound)) != 0) {
      float mp0 = -INFINITY, mp1 = -INFINITY;
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        mp0 = max3f(mp0, s_cur[e / 16][e % 16], s_cur[e / 16][e % 16 + 1]);
        mp1 = max3f(mp1, s_cur[e / 16][e % 16 + 2], s_cur[e / 16][e % 16 + 3]);
      }
      float mx = max3f(mp0, mp1, mp1);
      mx = max3f(mx, __shfl_xor(mx, 32, kWave), mx);
      const float tmax = mx * scale_log2;
      const bool grow = tmax > m_ref + kLazyRescale;
      rescale = __builtin_amdgcn_ballot_w64(grow) != 0;
      const float nref = grow ? tmax : m_ref;
      alpha = (m_ref == -INFINITY) ? 0.f : fast_exp2(m_ref - nref);
      m_ref = nref;
      ref = (nref == -INFINITY) ? 0.f : nref;
      psum = 0.f;
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        pw[e / 2] = pack_bf16x2(fast_exp2(fmaf(s_cur[e / 16][e % 16], scale_log2, -ref)),
                                fast_exp2(fmaf(s_cur[e / 16][e % 16 + 1], scale_log2, -ref)));
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
    // the exponents of this phase's gathers, and the block ids of the next one's
    if (kQK) {
      k_exps = exps_of(new_k);
      v_exps = exps_of(new_v);
      v_id = new_v;
      idsK = {{-1, -1, -1, -1}};
      idK = -1;
      if (i + 4 < N) {
        idsK = step_ids(i + 4);
        idK = my_entry(i + 4);
      }
      if (i + 2 < N) idV = my_entry(i + 2);
    }
    __syncthreads();
    if (rescale) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) oacc[dt] *= alpha;
    }
    bits >>= 4;
  };

  // Before the first phase: K of the first two steps converted, K of the third and
  // V of the first on their way.
  auto prologue = [&]() __attribute__((always_inline)) {
    bits = id_bits(step_ids(i0));
    if (i0 + 1 < N) bits |= id_bits(step_ids(i0 + 1)) << 4;
    if (i0 + 2 < N) bits |= id_bits(step_ids(i0 + 2)) << 8;
    const int a = real(my_entry(i0)), b = i0 + 1 < N ? real(my_entry(i0 + 1)) : -1;
    const int c2 = i0 + 2 < N ? real(my_entry(i0 + 2)) : -1;
    if (i0 + 3 < N) {
      idsK = step_ids(i0 + 3);
      idK = my_entry(i0 + 3);
    }
    idV = b;
    rk = gather(a, tiles.k_off);
    rv = gather(b, tiles.k_off);
    const uint32_t ea = exps_of(a), eb = exps_of(b);
    k_exps = exps_of(c2);
    v_exps = ea;
    v_id = a;
    convert_k(i0, ea);
    rk = rv;
    convert_k(i0 + 1, eb);
    rk = gather(c2, tiles.k_off);
    rv = gather(a, tiles.v_off);
  };

  if (N > i0) prologue();

  // A wavefront none of whose rows lies in the chunk (a short chunk's last
  // tile) still gathers and converts its share and meets every barrier, step for
  // step like the others, but does no matrix or softmax work and writes nothing.
  if (idle) {
    if (N > i0) {
      __syncthreads();
      __syncthreads();   // the others' q.k of the first step
      for (int i = i0; i < N; ++i) {
        convert_k(i + 2, k_exps);
        convert_v(i, v_id, v_exps);
        if (i + 1 < N) {
          const int new_k = real(idK), new_v = real(idV);
          rk = gather(new_k, tiles.k_off);
          rv = gather(new_v, tiles.v_off);
          k_exps = exps_of(new_k);
          v_exps = exps_of(new_v);
          v_id = new_v;
          idK = i + 4 < N ? my_entry(i + 4) : -1;
          if (i + 2 < N) idV = my_entry(i + 2);
        }
        __syncthreads();
      }
    }
    return;
  }

  if (N > i0) {
    __syncthreads();
    qk(i0, sA);
    __syncthreads();   // K of the first step is read; its pipeline step writes its buffer
    constexpr std::true_type T{};
    constexpr std::false_type F{};
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    if (i0 + 1 < N)
      phase(T, F, even, i0, sA, sB, pB, pA);
    else
      phase(F, F, even, i0, sA, sB, pB, pA);
    int i = i0 + 1;   // i0 is even: even steps use sA and pA
    for (; i + 1 <= N - 2; i += 2) {
      phase(T, T, odd, i, sB, sA, pA, pB);
      phase(T, T, even, i + 1, sA, sB, pB, pA);
    }
    if (i <= N - 2) {
      phase(T, T, odd, i, sB, sA, pA, pB);
      ++i;
    }
    // The last step, in one form whatever its parity (as two, the registers of both
    // would be live together).
    if (i0 + 1 < N) {
      if (i & 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) sA[k] = sB[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) pB[k] = pA[k];
      }
      phase(F, T, i & 1, i, sA, sB, pB, pA);
    }
    pv(N - 1, pA);   // its V was converted in the last phase
  }

  // ---- write O (this lane: row lm): normalised, or the item's partial ----
  {
    if (N <= i0) __syncthreads();   // no step has published lds.end
    const auto end = lds.end;
    const int n = end.n, cu0 = end.cu0, qstride = end.qstride;
    const float lt = l_run + __shfl_xor(l_run, 32, kWave);
    const int r = row0 + lm;
    if (__builtin_amdgcn_readfirstlane(end.slot) < 0) {
      // A lane holds 8-byte pieces of its row, two lanes per row: stored like
      // that, an instruction touches 32 rows of 16 bytes. Half the dims at a
      // time go through the wavefront's part of the K buffers and more,
      // which nobody reads any more, and are stored in runs of 128 bytes. A call, stored directly and
      // like this: 7 fresh prompts of 188 to 2031 rows (64 query heads over 8)
      // 172 -> 159 us, 64 of 100 rows (32 over 8) 59 -> 51 us, 4 of 64 rows 12.8 ->
      // 10.6 us; tiles of hundreds of steps do not notice.
      constexpr int kHalf = kD / 2, kRowBytes = kHalf * 2 + 16;   // padded against conflicts
      static_assert(kWaves * 32 * kRowBytes <= (int)(sizeof(lds.k) + sizeof(lds.more)), "fits");
      uint8_t* stage = &lds.k[0][0][0] + wave * 32 * kRowBytes;
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
          const uint2 w = *reinterpret_cast<const uint2*>(stage + rr * kRowBytes + sc * 8);
          if (row0 + rr < n)
            *reinterpret_cast<uint2*>(end.out + (size_t)(cu0 + row0 + rr) * qstride +
                                      (wave % G) * kD + half * kHalf + sc * 4) = w;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    } else if (r < n) {
      uint8_t* slot = end.slots + (size_t)end.slot * end.num_kv_heads * kSlotBytes;
      float2* po = reinterpret_cast<float2*>(slot) + wave * 32 * (kD / 2) + lm;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int a = 0; a < 8; ++a)   // dims dt 32 + (a / 2) 8 + lh 4 + (a % 2) 2 .. + 2
          po[(dt * 16 + (a / 2) * 4 + lh * 2 + a % 2) * 32] =
              make_float2(oacc[dt][2 * a], oacc[dt][2 * a + 1]);
      if (lh == 0)
        reinterpret_cast<float2*>(slot + kSlotFloats * sizeof(float))[wave * 32 + lm] =
            make_float2(m_ref, lt);
    }
  }
}

// One item of a one-row sequence: the eight wavefronts share its tokens evenly
// in whole steps of 64 and merge their states through LDS.
template <int G>
__device__ __forceinline__ void prefill_row_fp8(
    const PrefillItem& it, int g, const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
    int num_blocks, const int* __restrict__ block_table, uint16_t* __restrict__ out,
    uint8_t* __restrict__ row_slots, int num_q_heads, int num_kv_heads, int max_blocks,
    float scale_log2) {
  __shared__ __attribute__((aligned(16))) float o_lds[kWaves][G * kD];
  __shared__ float2 ml_lds[kWaves][G];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.i0, i1 = it.i1;
  const int per = max(1, (i1 - i0 + kWaves * kKeys - 1) / (kWaves * kKeys)) * kKeys;
  const int parts = (i1 - i0 + per - 1) / per;     // wavefronts with tokens
  const Fp8Tiles tiles(kv, num_kv_heads, kD, g);
  const size_t row = ((size_t)it.cu0 * num_q_heads + g * G) * kD;
  if (wave < parts) {
    const int t0 = i0 + wave * per;
    walk_fp8<kD, G, false>(tiles, q + row, block_table + (size_t)it.s * max_blocks, num_blocks, t0,
                           min(i1, t0 + per), scale_log2, o_lds[wave], ml_lds[wave]);
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

// One workgroup per (item of the plan, or tile of the tile map without one; kv
// head). kRows: the plan may hold one-row sequences.
template <int G, bool kRows>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads),
                          amdgpu_waves_per_eu(2, 2)))
void prefill_fp8_kernel(const uint16_t* __restrict__ q, const uint8_t* __restrict__ kv,
                        int num_blocks, const int* __restrict__ block_table,
                        const int* __restrict__ seq_lens, const int* __restrict__ cu,
                        uint16_t* __restrict__ out, PrefillLaunch l, int total_q, int num_q_heads,
                        int num_kv_heads, int max_blocks, int max_seq_len, float scale_log2) {
  constexpr int kRowsPerTile = 32 * kWaves / G;
  const int g = blockIdx.x % num_kv_heads;
  const int ti = blockIdx.x / num_kv_heads;
  PrefillItem it;
  if (kRows || l.head) {
    it = l.items[ti];   // the list has room for the whole grid: read beside the count
    if (ti >= l.head->items) return;
  } else {              // no plan: the tile map's whole tiles
    if (ti >= *l.tile_count) return;
    const int2 tl = l.tiles[ti];
    const int2 rows = chunk_rows(cu, tl.x, total_q);
    it.s = tl.x;
    it.q0 = tl.y;
    it.cu0 = rows.x;
    it.n = rows.y - rows.x;
    it.L = min(max(seq_lens[tl.x], 0), min(max_seq_len, max_blocks * kBS));
    const int last_pos = min(it.L - it.n + it.q0 + min(kRowsPerTile, it.n - it.q0) - 1, it.L - 1);
    it.i0 = 0;
    it.i1 = last_pos >= 0 ? last_pos / kKeys + 1 : 0;
    it.slot = -1;
  }
  if (kRows && it.q0 < 0)
    prefill_row_fp8<G>(it, g, q, kv, num_blocks, block_table, out, l.row_slots, num_q_heads,
                       num_kv_heads, max_blocks, scale_log2);
  else
    prefill_tile_fp8<G>(it, g, q, kv, num_blocks, block_table, out, l.slots, num_q_heads,
                        num_kv_heads, max_blocks, scale_log2);
}

template <int G>
static hipError_t launch_prefill_fp8_t(const PrefillArgs& a, const PrefillLaunch& l, bool rows) {
  auto kernel = l.head && rows ? prefill_fp8_kernel<G, true> : prefill_fp8_kernel<G, false>;
  hipLaunchKernelGGL(kernel, dim3(l.blocks), dim3(kThreads), 0, a.stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint8_t*>(a.kv),
                     a.num_blocks, a.block_table, a.seq_lens, a.cu_seqlens_q,
                     static_cast<uint16_t*>(a.out), l, a.total_q_tokens, a.num_q_heads,
                     a.num_kv_heads, a.max_blocks, a.max_seq_len, a.scale * kLog2e);
  return hipGetLastError();
}

hipError_t launch_prefill_fp8(const PrefillArgs& a, const PrefillLaunch& l) {
  const bool rows = a.num_seqs > 1 || a.total_q_tokens == 1;   // may hold one-row sequences
  switch (a.num_q_heads / a.num_kv_heads) {
    case 1: return launch_prefill_fp8_t<1>(a, l, rows);
    case 2: return launch_prefill_fp8_t<2>(a, l, rows);
    case 4: return launch_prefill_fp8_t<4>(a, l, rows);
    case 8: return launch_prefill_fp8_t<8>(a, l, rows);
    default: return hipErrorNotSupported;
  }
}

}  // namespace kvattn
