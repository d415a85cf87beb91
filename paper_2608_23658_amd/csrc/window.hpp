// Which keys, blocks and steps a window leaves, in plain arithmetic that the host runs too.
// What lies in blocks wholly before the first key that is seen may be given up by the caller,
// its memory with it, whatever the block table still says of it: walks begin at a block.
#pragma once

namespace kvattn {

constexpr int kNoWindow = 0x3fffffff;

// First key that the row at position pos sees.
constexpr int first_key(int pos, int window) {
  return pos - window + 1 > 0 ? pos - window + 1 : 0;
}

// Where a walk for rows from position pos on begins: with the block of the first key.
constexpr int walk_start(int pos, int window) { return first_key(pos, window) & ~15; }

// Steps of 64 keys from walk_start(pos, window) on that reach the last row, at position last
// (below 0: no row sees a key).
constexpr int walk_steps(int pos, int last, int window) {
  return last >= 0 ? (last - walk_start(pos, window)) / 64 + 1 : 0;
}

}  // namespace kvattn
