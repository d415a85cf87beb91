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
// Rounding is the scaled conversion's, two values an instruction: to nearest even at
// every scale, subnormal codes included (checked over all bf16 values and exponents); past
// the largest code it gives NaN, so where a value can get there (the largest exponent) a
// slower form clamps first.
//
// A workgroup of four wavefronts has the runs that begin in a window of the list.
// A window of 32 tokens of a chunk is two runs, K and V of each a wavefront's; the tokens of a
// decode step are a run each, and a window of 2 spreads them over the CUs. Only the
// device knows which it is, so the window goes by the number of tokens. bf16, 8 heads of
// 128 (rocprof, us), windows of 2 / 8 / 32:
//   tokens            256               512              2048              8192
//   one a block   5.3 / 8.2 / 22.9  7.8 / 9.0 / 23.2  22.6 / 19.5 / 27.0  88 / 71 / 72
//   one chunk     4.2 / 3.8 /  5.0  5.2 / 4.1 /  5.0  12.3 /  6.8 /  5.8  39 / 17 / 11.5
// A list that holds both pays for it: 2048 in order 6.3 us, with 128 one a block behind them
// 24.2; 256 one a block in a list padded to 8192 23.1.
// A chunk of 8192 moves 50 MB, 10.6 us at the rate of a large copy. A token alone
// touches all 16 lines of its V tile, 4 tokens x 4 dims to 16 bytes, with a byte each.

#include "append_fp8.hpp"
#include "launch.hpp"

namespace kvattn {

template <int ESZ, int D, int kWin>
__global__ __launch_bounds__(kAppendWaves * kWave) void kv_append_fp8_kernel(
    const uint8_t* __restrict__ k_new, const uint8_t* __restrict__ v_new,
    const int* __restrict__ slot_mapping, uint8_t* __restrict__ kv, int num_tokens,
    int num_kv_heads, int capacity) {
  const size_t stride = (size_t)num_kv_heads * (D * ESZ);
  append_fp8<ESZ, D, kWin>(blockIdx.x, k_new, stride, v_new, stride, slot_mapping, kv, num_tokens,
                           num_kv_heads, capacity, NoPrep{});
}

template <int ESZ, int D>
static hipError_t launch_append_fp8_t(const AppendArgs& a) {
  const int win = append_window(a.num_tokens);
  const long long blocks = ((long long)a.num_tokens + win - 1) / win * a.num_kv_heads;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  auto kernel = win == kFewWindow    ? kv_append_fp8_kernel<ESZ, D, kFewWindow>
                : win == kSomeWindow ? kv_append_fp8_kernel<ESZ, D, kSomeWindow>
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
