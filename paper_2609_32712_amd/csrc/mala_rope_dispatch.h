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

// A wavefront of the block-scaled write takes the blocks that begin among `chunk` tokens, of `heads`
// heads of K or of V.
constexpr int kBlockChunk = 16;
struct BlockWritePlan {
  int chunk, heads;
  int64_t waves;
};
inline BlockWritePlan block_write_plan(int T, int Hkv, bool rope) {
  BlockWritePlan x;
  x.chunk = std::clamp(T / 256, 1, kBlockChunk);
  const int64_t chunks = ((int64_t)T + x.chunk - 1) / x.chunk;
  const int64_t parts = std::clamp<int64_t>(4 * 4 * kNumCus / chunks, 1, Hkv);
  x.heads = (int)((Hkv + parts - 1) / parts);
  x.waves = chunks * 2 * ((Hkv + x.heads - 1) / x.heads);
  return x;
}

}  // namespace mala
