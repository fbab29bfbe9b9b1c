// Rows into pages of e4m3 values with a scale per block of 16 rows and KV head, and the rotation of
// a step's queries and keys in the same launch (gfx950).
//
// A block's scale is 2^e.  e of new rows is the least integer with amax <= 448 2^e (finite values
// alone), kept in [kScaleMin, kScaleMax]; a block whose row 0 is new starts anew, any other one
// takes the larger of its e and the new one, and when that grows its other rows are rounded again,
// to nearest even as the new ones.  Scales are powers of two so that this second rounding is exact
// but where a value leaves the normal range, and so that value x scale is a bf16.
//
// What bounds it: HBM (2 bytes read and 1 written per value); small calls the chain slots -> rows
// -> stores.
#include "mala_rope.h"

namespace mala {

namespace {

constexpr int kWindow = 63;    // tokens of a block lie at most so far apart

// e of a block whose largest |value| is the bf16 with these bits (finite): 448 = 1.75 x 2^8.
__device__ __forceinline__ int block_exponent(uint32_t bf16_bits) {
  return min(max((int)(((bf16_bits << 16) + 0x1fffffu) >> 23) - 127 - 8, kScaleMin), kScaleMax);
}
__device__ __forceinline__ float power_of_two(int e) {     // e in [-126, 127]
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}
// The larger of the maximum `m` and the finite |values| of two bf16 pairs' bits
__device__ __forceinline__ uint32_t max_finite(uint32_t m, uint32_t u) {
  uint32_t lo = u & 0x7fffu, hi = u & 0x7fff0000u;
  lo = lo >= 0x7f80u ? 0 : lo;
  hi = hi >= 0x7f800000u ? 0 : hi;
  return max_u16x2(m, lo | hi);
}

// e4m3 bytes of four values over a scale, at most +-limit (NaN stays)
__device__ __forceinline__ int to_block4(float a, float b, float c, float d, float inv, float limit) {
  const auto lim = [&](float x) {
    x *= inv;
    return x != x ? x : fminf(fmaxf(x, -limit), limit);
  };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lim(a), lim(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(lim(c), lim(d), r, true);
}
__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// The n-th set bit of mask.
__device__ __forceinline__ int set_bit(uint64_t mask, int n) {
  for (int i = 0; i < n; ++i) mask &= mask - 1;
  return __builtin_ctzll(mask);
}

// Keys and values of the blocks whose first token (of this call) is among the chunk's tokens.
// LPR lanes take a block of one head, all its rows in registers.
template <int D, bool ROPE>
struct BlockWriter {
  static constexpr int LPR = D / 16, SUBS = 256 / LPR;
  static constexpr int G = ROPE ? 256 / D : kBlockChunk;    // blocks at a time (their angles in LDS)

  struct Shared {
    int window[kBlockChunk + 2 * kWindow];
    __attribute__((aligned(16))) int rows[kBlockChunk][16];   // token of each row, or -1
    int block[kBlockChunk];
    __attribute__((aligned(16))) f32x2 turns[ROPE ? G : 1][ROPE ? 16 : 1][ROPE ? D / 2 : 1];
  };

  static __device__ __forceinline__ void run(const PagedWriteParams& p, const Turn& turn, unsigned group,
                                             Shared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = (int)group * p.chunk, Hkv = p.c.Hkv;
    const int slots = (int)(p.c.num_pages * (unsigned)p.c.page_size);
    // which tokens share a block
    for (int j = tid; j < p.chunk + 2 * kWindow; j += 256) {
      const int t = t0 - kWindow + j;
      int s = t >= 0 && t < p.T ? p.slots[t] : -1;
      sh.window[j] = s < slots ? s : -1;
    }
    __syncthreads();
    for (int ci = w; ci < p.chunk; ci += 4) {
      const int mine = sh.window[kWindow + ci], block = mine >> 4;
      const int before = lane < kWindow ? sh.window[kWindow + ci - 1 - lane] : -1;
      const int after = sh.window[kWindow + ci + lane];
      const bool first = mine >= 0 && !wave_any(before >= 0 && before >> 4 == block);
      if (lane < 16) sh.rows[ci][lane] = -1;
      if (first && after >= 0 && after >> 4 == block) sh.rows[ci][after & 15] = t0 + ci + lane;
      if (lane == 0) sh.block[ci] = first ? block : -1;
    }
    __syncthreads();
    const uint64_t firsts =
        __builtin_amdgcn_ballot_w64(lane < p.chunk && sh.block[lane < p.chunk ? lane : 0] >= 0);
    const int n = __builtin_popcountll(firsts);
    for (int g0 = 0; g0 < n; g0 += G) {
      const int here = min(G, n - g0);
      if constexpr (ROPE) {
        const int pairs = turn.R / 2;
        if (g0) __syncthreads();
        for (int i = tid; i < here * 16 * pairs; i += 256) {
          const int row = i / pairs, pair = i - row * pairs;
          const int t = sh.rows[set_bit(firsts, g0 + row / 16)][row & 15];
          if (t < 0) continue;
          float c, s;
          turn_of(turn.pos ? turn.pos[t] : t, turn.inv_freq[pair], turn.scale, turn.sin_scale, c, s);
          sh.turns[row / 16][row & 15][pair] = f32x2{c, s};
        }
        __syncthreads();
      }
      for (int u = tid / LPR; u < here * 2 * Hkv; u += SUBS) {
        const int g = u / (2 * Hkv), kind = (u - g * 2 * Hkv) / Hkv, h = u - (2 * g + kind) * Hkv;
        write_block(p, turn, sh, set_bit(firsts, g0 + g), g, kind, h);
      }
    }
  }

  static __device__ __forceinline__ void write_block(const PagedWriteParams& p, const Turn& turn, Shared& sh,
                                                     int ci, int g, int kind, int h) {
    const int lr = threadIdx.x % LPR;
    const unsigned per_page = (unsigned)p.c.page_size / kPageRows, block = sh.block[ci];
    const unsigned page = block / per_page, within = block - page * per_page;
    const bool keys = ROPE && kind == 0;
    const Pieces pc = pieces_of(lr, keys ? turn.R : 0, keys ? turn.interleaved : 1);
    const char* in = (kind ? p.v : p.k) + h * p.head_stride;
    char* out = (kind ? p.c.v : p.c.k) + (int64_t)page * p.c.page_stride + h * p.c.head_stride +
                (int64_t)(within * kPageRows) * p.c.token_stride;
    uint8_t* scale = (kind ? p.c.vb : p.c.kb) + ((int64_t)page * p.c.Hkv + h) * per_page + within;
    int t[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = sh.rows[ci][r];
    const int held = t[0] >= 0 ? kScaleMin : min(max((int)*scale - 127, kScaleMin), kScaleMax);

    i32x4 x[16][2];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r][0] = x[r][1] = i32x4{0, 0, 0, 0};
      if (t[r] >= 0) {
        const char* row = in + t[r] * p.token_stride;
        x[r][0] = *reinterpret_cast<const i32x4*>(row + pc.first * 16);
        x[r][1] = *reinterpret_cast<const i32x4*>(row + pc.second * 16);
      }
    }
    if (ROPE && pc.turned) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (t[r] < 0) continue;
        float v[16], c[8], s[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            v[8 * half + 2 * i] = bf16_lo((uint32_t)x[r][half][i]);
            v[8 * half + 2 * i + 1] = bf16_hi((uint32_t)x[r][half][i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const f32x2 a = sh.turns[g][r][8 * lr + i];
          c[i] = a[0];
          s[i] = a[1];
        }
        turn_pieces(v, c, s, turn.interleaved);
        x[r][0] = to_bf16x8(v);        // the key as it would be stored without a cache
        x[r][1] = to_bf16x8(v + 8);
      }
    }
    uint32_t most = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        most = max_finite(max_finite(most, (uint32_t)x[r][0][i]), (uint32_t)x[r][1][i]);
    most = max(most & 0xffffu, most >> 16);
    // over the LPR lanes of the block
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xf, 0xf, true));   // lane ^ 1
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xf, 0xf, true));   // lane ^ 2
    if constexpr (LPR == 8)   // row_half_mirror: the other four of eight
      most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x141, 0xf, 0xf, true));
    const int e = max(held, block_exponent(most));
    if (lr == 0) *scale = (uint8_t)(e + 127);

    // (448 x 2^120 is no bf16 any more)
    const float inv = power_of_two(-e), limit = e == kScaleMax ? 240.f : 448.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (t[r] < 0) continue;
      i32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = (uint32_t)x[r][i / 2][2 * (i % 2)], b = (uint32_t)x[r][i / 2][2 * (i % 2) + 1];
        y[i] = to_block4(bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b), inv, limit);
      }
      char* row = out + r * p.c.token_stride;
      *reinterpret_cast<i32x2*>(row + pc.first * 8) = i32x2{y[0], y[1]};
      *reinterpret_cast<i32x2*>(row + pc.second * 8) = i32x2{y[2], y[3]};
    }
    // a larger scale than the block had: its other rows
    if (t[0] < 0 && e > held) {
      const float less = power_of_two(max(held - e, -100));
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (t[r] >= 0) continue;
        i32x4* row = reinterpret_cast<i32x4*>(out + r * p.c.token_stride + 16 * lr);
        i32x4 y = *row;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(y[i], false);
          const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(y[i], true);
          y[i] = to_block4(a[0], a[1], b[0], b[1], less, 448.f);
        }
        *row = y;
      }
    }
  }
};

template <int D>
__global__ __launch_bounds__(256) void mala_paged_block_write_kernel(PagedWriteParams p) {
  __shared__ typename BlockWriter<D, false>::Shared sh;
  BlockWriter<D, false>::run(p, Turn{}, blockIdx.x, sh);
}

// Keys and values into a block-scaled cache by the first workgroups, queries by the others.
template <int D>
__global__ __launch_bounds__(256) void mala_paged_block_rope_kernel(PagedRopeWriteParams p) {
  __shared__ typename BlockWriter<D, true>::Shared sh;
  if (blockIdx.x < p.kv_groups) {
    BlockWriter<D, true>::run(p.w, p.q.turn, blockIdx.x, sh);
  } else {
    const unsigned nx = (p.q.T + rope_tokens(D) - 1) / rope_tokens(D), i = blockIdx.x - p.kv_groups;
    turn_rows<D, false, false>(p.q, i % nx * rope_tokens(D), (int)(i / nx) * p.q.per);
  }
}

// The same for a cache of bf16, or of e4m3 with a scale per head: every row is its own.
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void mala_paged_rope_write_kernel(PagedRopeWriteParams p) {
  constexpr int LPR = D / 16, TOK = rope_tokens(D);
  const unsigned nx = (p.q.T + TOK - 1) / TOK;
  if (blockIdx.x >= p.kv_groups) {
    const unsigned i = blockIdx.x - p.kv_groups;
    turn_rows<D, false, false>(p.q, i % nx * TOK, (int)(i / nx) * p.q.per);
    return;
  }
  const PagedWriteParams& w = p.w;
  const Turn& turn = p.q.turn;
  const unsigned t = blockIdx.x % nx * TOK + threadIdx.x / LPR, P = w.c.page_size;
  if (t >= p.q.T) return;
  const int slot = w.slots[t], lr = threadIdx.x % LPR;
  if (slot < 0 || (unsigned)slot >= w.c.num_pages * P) return;
  const unsigned page = slot / P, row = slot - page * P;
  const int kind = blockIdx.x / nx % 2, h0 = blockIdx.x / nx / 2 * w.chunk;
  const Pieces pc = pieces_of(lr, kind ? 0 : turn.R, turn.interleaved);
  float c[8], s[8];
  if (pc.turned) {
    const int pos = turn.pos ? turn.pos[t] : (int)t;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      turn_of(pos, turn.inv_freq[8 * lr + k], turn.scale, turn.sin_scale, c[k], s[k]);
  }
  for (int h = h0; h < min(h0 + w.chunk, w.c.Hkv); ++h) {
    const char* x = (kind ? w.v : w.k) + t * w.token_stride + h * w.head_stride;
    char* out = (kind ? w.c.v : w.c.k) + page * w.c.page_stride + h * w.c.head_stride + row * w.c.token_stride;
    float v[16];
    load_piece<false>(x + pc.first * 16, v);
    load_piece<false>(x + pc.second * 16, v + 8);
    if (pc.turned) turn_pieces(v, c, s, turn.interleaved);
    const float* scales = kind ? w.c.vs : w.c.ks;
    const float scale = E4M3 && scales ? scales[h] : 1.f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int piece = half ? pc.second : pc.first;
      const i32x4 y = to_bf16x8(v + 8 * half);     // (a value as it is, a rotated key rounded)
      if constexpr (E4M3) {
        int e[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t a = (uint32_t)y[2 * i], b = (uint32_t)y[2 * i + 1];
          e[i] = to_e4m3x4(bf16_lo(a) / scale, bf16_hi(a) / scale, bf16_lo(b) / scale, bf16_hi(b) / scale);
        }
        *reinterpret_cast<i32x2*>(out + piece * 8) = i32x2{e[0], e[1]};
      } else {
        *reinterpret_cast<i32x4*>(out + piece * 16) = y;
      }
    }
  }
}

}  // namespace

hipError_t launch_paged_block_write(PagedWriteParams p, int D, hipStream_t st) {
  p.chunk = block_write_chunk(p.T);
  const dim3 grid((unsigned)((p.T + p.chunk - 1) / p.chunk));
  if (D == 128)
    hipLaunchKernelGGL(mala_paged_block_write_kernel<128>, grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(mala_paged_block_write_kernel<64>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

template <int D>
static void launch_rope_write_t(PagedRopeWriteParams& p, hipStream_t st) {
  const unsigned nx = (p.q.T + rope_tokens(D) - 1) / rope_tokens(D);
  unsigned q_groups = 0;
  if (p.q.r[0].H) {
    p.q.per = rope_heads_per_group(p.q.T, p.q.r[0].H, D);
    q_groups = nx * ((p.q.r[0].H + p.q.per - 1) / p.q.per);
  }
  if (p.w.c.fmt == kCacheBlock) {
    p.w.chunk = block_write_chunk(p.w.T);
    p.kv_groups = (p.w.T + p.w.chunk - 1) / p.w.chunk;
    hipLaunchKernelGGL(mala_paged_block_rope_kernel<D>, dim3(p.kv_groups + q_groups), dim3(256), 0, st, p);
    return;
  }
  p.w.chunk = rope_heads_per_group(p.w.T, p.w.c.Hkv, D);        // heads at a time
  p.kv_groups = nx * 2 * ((p.w.c.Hkv + p.w.chunk - 1) / p.w.chunk);
  if (p.w.c.fmt == kCacheE4M3)
    hipLaunchKernelGGL((mala_paged_rope_write_kernel<D, true>), dim3(p.kv_groups + q_groups), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((mala_paged_rope_write_kernel<D, false>), dim3(p.kv_groups + q_groups), dim3(256), 0, st, p);
}

hipError_t launch_paged_rope_write(PagedRopeWriteParams p, int D, hipStream_t st) {
  D == 128 ? launch_rope_write_t<128>(p, st) : launch_rope_write_t<64>(p, st);
  return hipGetLastError();
}

}  // namespace mala
