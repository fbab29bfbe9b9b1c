// How rotations and block-scaled writes are shared out: launch rules, plain C++ (the tests compile
// them for the CPU).
#pragma once
#include <stdint.h>

#include <algorithm>

#include "mala_dispatch.h"

namespace mala {

// Tokens of a workgroup of 256 threads, D / 16 lanes a row.
constexpr int rope_tokens(int D) { return 256 / (D / 16); }

// Heads that a workgroup of the rotation takes for its tokens.
inline int rope_heads_per_group(unsigned tokens, int heads, int D) {
  const long groups = (tokens + rope_tokens(D) - 1) / rope_tokens(D);
  const long slices = std::min<long>(heads, std::max<long>(1, 8 * kNumCus / groups));
  return (int)((heads + slices - 1) / slices);
}

// Tokens that a workgroup of the block-scaled write looks at.
constexpr int kBlockChunk = 32;
inline int block_write_chunk(int T) { return std::clamp(T / 1024, 1, kBlockChunk); }

}  // namespace mala
