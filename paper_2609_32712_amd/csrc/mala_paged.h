// Parameter blocks and launchers of the paged KV cache kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mala_device.h"
#include "mala_paged_dispatch.h"
#include "mala_rope_dispatch.h"

namespace mala {

constexpr int kPageRows = 16;   // page sizes are multiples of this: 16 rows from a multiple of
                                // 16 on lie in one page, so they share one base address

// What a cache holds: bf16; e4m3 with a scale per KV head; e4m3 with a scale 2^e for each block of
// kPageRows rows and KV head, e + 127 a byte in [127 + kScaleMin, 127 + kScaleMax] (others read as
// the nearer of the two): value x scale is then a bf16 that is no subnormal, and finite.
enum { kCacheBf16 = 0, kCacheE4M3 = 1, kCacheBlock = 2 };
constexpr int kScaleMin = -117, kScaleMax = 120;

// Pages of K and V: row r of page i, KV head h at byte i * page_stride + h * head_stride +
// r * token_stride of k and v.  Strides in bytes (multiples of 16).
struct PagedCache {
  char* k;
  char* v;
  const float* ks;   // [Hkv] e4m3 scales, or null (1)
  const float* vs;
  uint8_t* kb;       // [num_pages, Hkv, page_size / kPageRows] exponents of a kCacheBlock
  uint8_t* vb;
  int64_t page_stride, head_stride, token_stride;
  int num_pages, page_size, Hkv;
  int fmt;           // kCache*
};

struct PagedUpdateParams {
  const int32_t* lens;
  const int32_t* new_lens;
  int32_t* table;
  int32_t* ring;
  const int32_t* state;
  int32_t* lens_out;
  int32_t* cu;
  int32_t* slots;
  int32_t* positions;   // or null
  int32_t* state_out;
  int R, W, P, num_pages, C, max_tokens;
};

struct PagedWriteParams {
  PagedCache c;
  const char* k;        // bf16 rows: token t, head h at byte t * token_stride + h * head_stride
  const char* v;
  int64_t token_stride, head_stride;
  const int32_t* slots;
  int T;
  int chunk, units;     // tokens and heads at a time (see block_write_plan), set by the launch
};

struct PagedReadParams {
  PagedCache c;
  const int32_t* table;
  const int32_t* cu;
  char* k;              // bf16 [Hkv, total, D]
  char* v;
  int S, W, max_len, total;
};

struct PagedDecParams {
  PagedCache c;
  const __bf16* q;
  const int32_t* table;
  const int32_t* lens;
  int2* plan;           // [B]: number of a sequence's first block, its blocks
  float* part;          // [nblk, Hq, D + kDecStride], blocks of all sequences in order
  void* o;              // fp32, or bf16 when o_bf16
  int o_bf16;
  float* lse;
  int32_t* head_tiles;  // or null
  unsigned long long* counters;
  int B, Hq, W, max_len;
  int unit;             // tiles per split (tau = 0: 1)
  int target, ragged;   // blocks that the tiles are shared out to, and of sequences of unequal length
  int min_tpw;          // tiles per wavefront at least
  int nblk;             // blocks of all sequences at most
  int sorted;           // whether they are dealt in the order of their sizes
  int nchunk;           // ceil((Hq / Hkv) / 16)
  float scale2, log2tau;
};

// e4m3 bytes of 4 fp32 values (nearest even; beyond +-448 the largest finite value, NaN stays)
__device__ __forceinline__ int to_e4m3x4(float a, float b, float c, float d) {
  const auto lim = [](float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lim(a), lim(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(lim(c), lim(d), r, true);
}

// 2^e of a block's byte, as an fp32's bits
__device__ __forceinline__ uint32_t block_scale_bits(uint32_t byte) {
  return min(max(byte, 127u + kScaleMin), 127u + kScaleMax) << 23;
}

// Inclusive sum over the wavefront's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15 to rows 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31 to rows 2, 3
  return x;
}

// Maximum over the wavefront's lanes of x >= 0.
__device__ __forceinline__ int wave_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}

hipError_t launch_paged_update(const PagedUpdateParams& p, hipStream_t st);
hipError_t launch_paged_write(const PagedWriteParams& p, int D, hipStream_t st);
hipError_t launch_paged_block_write(PagedWriteParams p, int D, hipStream_t st);
hipError_t launch_paged_read(const PagedReadParams& p, int D, hipStream_t st);
hipError_t launch_paged_decode(PagedDecParams p, int D, int split_tokens, hipStream_t st);

}  // namespace mala
