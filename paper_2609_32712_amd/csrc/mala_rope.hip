// Rotary positions of queries and keys, and of their gradients (gfx950).
//
// Every row is read and written once, so HBM bounds a large call: 5.7-5.9 TB/s of reads and writes
// (16000 tokens of 32 + 8 heads in bf16 55 us, their fp32 gradients to bf16 85), as much as a copy
// kernel; an angle is computed once per token and pair and kept for the heads that a workgroup takes.
// Small calls are latency alone (64 tokens 3.1 us).
#include "mala_rope.h"

namespace mala {

namespace {

template <int D, bool IN32, bool OUT32, bool INTER, bool ONCE>
__global__ __launch_bounds__(256) void mala_rope_kernel(RopeParams p) {
  // consecutive workgroups: the tokens of some heads, or (heads_first) the heads of some tokens
  const unsigned slices = gridDim.y, i = blockIdx.x + blockIdx.y * gridDim.x;
  if (p.heads_first)
    turn_rows<D, IN32, OUT32, INTER, ONCE, 1>(p, i / slices * rope_tokens(D), i % slices * p.per);
  else
    turn_rows<D, IN32, OUT32, INTER, ONCE, 1>(p, blockIdx.x * rope_tokens(D), blockIdx.y * p.per);
}

template <int D, bool IN32, bool OUT32, bool INTER>
void launch_l(const RopeParams& p, hipStream_t st) {
  const int heads = p.r[0].H + p.r[1].H;
  const dim3 grid((p.B * p.T + rope_tokens(D) - 1) / rope_tokens(D), (heads + p.per - 1) / p.per);
  if constexpr (D == 128)
    if (rope_loads_once(p.B * p.T, heads, D, p.turn.R, IN32 ? 4 : 2)) {
      hipLaunchKernelGGL((mala_rope_kernel<D, IN32, OUT32, INTER, true>), grid, dim3(256), 0, st, p);
      return;
    }
  hipLaunchKernelGGL((mala_rope_kernel<D, IN32, OUT32, INTER, false>), grid, dim3(256), 0, st, p);
}
template <int D, bool IN32, bool OUT32>
void launch_t(const RopeParams& p, hipStream_t st) {
  p.turn.interleaved ? launch_l<D, IN32, OUT32, true>(p, st) : launch_l<D, IN32, OUT32, false>(p, st);
}
template <int D>
void launch_d(const RopeParams& p, bool in32, bool out32, hipStream_t st) {
  if (in32)
    out32 ? launch_t<D, true, true>(p, st) : launch_t<D, true, false>(p, st);
  else
    out32 ? launch_t<D, false, true>(p, st) : launch_t<D, false, false>(p, st);
}

}  // namespace

hipError_t launch_rope(RopeParams p, int D, bool in32, bool out32, hipStream_t st) {
  p.per = rope_heads_per_group(p.B * p.T, p.r[0].H + p.r[1].H, D);
  // What runs at one time should lie together.  us per call of 16000 tokens, tokens / heads first: out of
  // and into token-major rows 73.8 / 64.9, head-major ones 55.0 / 62.5, from one to the other 60.8 / 61.8.
  p.heads_first = p.r[0].xh < p.r[0].xt && p.r[0].oh < p.r[0].ot;
  D == 128 ? launch_d<128>(p, in32, out32, st) : launch_d<64>(p, in32, out32, st);
  return hipGetLastError();
}

}  // namespace mala
