// How rotations and block-scaled writes are shared out: launch rules, plain C++ (the tests compile
// them for the CPU).
#pragma once
#include <stdint.h>

#include <algorithm>

#include "mala_dispatch.h"

#ifndef MALA_HOST_DEVICE
#ifdef __HIP__
#define MALA_HOST_DEVICE __host__ __device__
#else
#define MALA_HOST_DEVICE
#endif
#endif

namespace mala {

// Tokens of a workgroup of 256 threads, D / 16 lanes a row.
constexpr int rope_tokens(int D) { return 256 / (D / 16); }

// Heads that a workgroup of the rotation takes for its tokens: fewer heads are more workgroups, each
// with the angles to compute again.  us per call with 4 / 8 / 16 / 32 workgroups per CU (32 + 8
// heads): 16000 tokens of D = 128 in bf16 56.6 / 58.9 / 57.3 / 54.9, their fp32 gradients to bf16 90.0 /
// 90.7 / 86.0 / 84.7; 32000 of D = 64 out of token-major rows 68.3 / 75.5 / 74.9 / 73.7, 20000 of 16 + 4
// heads 19.8 / 20.5 / 19.9 / 19.7.
inline int rope_heads_per_group(unsigned tokens, int heads, int D) {
  const long groups = (tokens + rope_tokens(D) - 1) / rope_tokens(D);
  const long slices = std::min<long>(heads, std::max<long>(1, (D == 128 ? 32 : 4) * kNumCus / groups));
  return (int)((heads + slices - 1) / slices);
}

// Whether rows are loaded past the caches: of inputs larger than half of the memory-side cache (256
// MB), which are not in it, where each load takes whole lines of 128 bytes.  us per call, through the
// caches / past them: gradients of 16000 tokens (fp32, 328 MB) 93.7 / 88.8, 16000 tokens in bf16 (164
// MB) 60.0 / 57.5; where only half of a line is taken at a time, half of each head turned 74.9 / 78.9,
// D = 64 74.9 / 79.6; and of 2000 tokens (20 MB) 9.7 / 10.8.
inline bool rope_loads_once(unsigned tokens, int heads, int D, int R, int size) {
  return D == 128 && R == D && (double)tokens * heads * D * size > 128e6;
}

// A workgroup of the block-scaled write takes the blocks that begin among `chunk` tokens, of K and V
// of some heads: `units` for each of its four wavefronts, a head of K or of V each.  Small calls want
// few tokens to a workgroup (one behind the other), large ones fewer workgroups that find no block's
// first token; with whole chunks a workgroup per some heads, or where keys are turned, angles
// computed for as many of them as possible.  us per call with 2 / 4 / 16 workgroups per CU: writes of
// 20000 tokens of 8 heads 22.3 / 22.3 / 20.7, of 2000 6.9 / 5.6 / 5.3, of 1000 decodes 5.1 / 4.8 / 6.3; turned
// 16000 tokens with 32 heads' queries 71.3 / 71.2 / 77.0, 512 decodes 5.7 / 7.1 / 7.1.
constexpr int kBlockChunk = 16;
struct BlockWritePlan {
  int chunk, units;
  int64_t groups;
};
MALA_HOST_DEVICE inline int block_write_parts(int Hkv, int units) { return (2 * Hkv + 4 * units - 1) / (4 * units); }
inline BlockWritePlan block_write_plan(int T, int Hkv, bool rope) {
  BlockWritePlan x;
  x.chunk = std::clamp(T / kNumCus, 1, kBlockChunk);
  const int64_t chunks = ((int64_t)T + x.chunk - 1) / x.chunk;
  const int64_t want = (x.chunk == kBlockChunk ? (rope ? 4 : 16) : rope ? 2 : 4) * kNumCus;
  const int64_t parts = std::clamp<int64_t>(want / chunks, 1, (2 * (int64_t)Hkv + 3) / 4);
  x.units = (int)((2 * (int64_t)Hkv + 4 * parts - 1) / (4 * parts));
  x.groups = chunks * block_write_parts(Hkv, x.units);
  return x;
}

}  // namespace mala
