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

// e of a block whose largest |value| is the bf16 with these bits (finite): 448 = 1.75 x 2^8.
__device__ __forceinline__ int block_exponent(uint32_t bf16_bits) {
  return min(max((int)(((bf16_bits << 16) + 0x1fffffu) >> 23) - 127 - 8, kScaleMin), kScaleMax);
}
__device__ __forceinline__ float power_of_two(int e) {     // e in [-126, 127]
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

typedef short s16x2 __attribute__((ext_vector_type(2)));
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

// Keys and values of the blocks whose first token (of this call) is among the wavefront's chunk of
// tokens, of some heads of K or of V.  No wavefront waits for another: each finds the rows of its
// blocks from the slots around its tokens, by ballots and a lane exchange.  D / 16 lanes a row.
template <int D, bool ROPE, bool INTER>
struct BlockWriter {
  static constexpr int LPR = D / 16, RPI = 64 / LPR, NI = kPageRows / RPI;   // rows at a time, times

  // `at`: the wavefront's number among those of the keys and values
  static __device__ __forceinline__ void run(const PagedWriteParams& p, const Turn& turn, unsigned at) {
    const int lane = threadIdx.x & 63;
    const int parts = (p.c.Hkv + p.heads - 1) / p.heads;      // of the heads, for K and for V
    const unsigned chunk = at / (2 * parts);
    const int part = at - chunk * 2 * parts, kind = part >= parts, h0 = (part - kind * parts) * p.heads;
    const int64_t t0 = (int64_t)chunk * p.chunk;
    if (t0 >= p.T) return;
    const int slots = (int)(p.c.num_pages * (unsigned)p.c.page_size);
    const auto slot_of = [&](int64_t t) {
      if (t < 0 || t >= p.T) return -1;
      const int s = p.slots[t];
      return s < slots && s >= 0 ? s : -1;
    };
    const int before = slot_of(t0 - 64 + lane), here = slot_of(t0 + lane);
    const int after = p.chunk > 1 ? slot_of(t0 + 64 + lane) : -1;
    uint64_t todo = __builtin_amdgcn_ballot_w64(here >= 0 && lane < p.chunk);
    while (todo) {
      const int ci = __builtin_ctzll(todo), first = __builtin_amdgcn_readlane(here, ci), block = first >> 4;
      // (-1 >> 4 is no block's number.  Tokens of a block lie within 64: those before from lane ci + 1 on,
      // those after below lane ci)
      const uint64_t same = __builtin_amdgcn_ballot_w64(here >> 4 == block);
      todo &= ~same;
      if (__builtin_amdgcn_ballot_w64(before >> 4 == block) >> ci >> 1) continue;
      const uint64_t more =
          p.chunk > 1 ? __builtin_amdgcn_ballot_w64(after >> 4 == block) & ((1ull << ci) - 1) : 0;
      // token of row r of the block, from t0 on, plus 1, in lane r < 16; 0 for none
      int token;
      if (!(same & (same - 1)) && !more) {
        token = lane == (first & 15) ? ci + 1 : 0;
      } else {
        // (of tokens with the same slot, one's number arrives)
        token = __builtin_amdgcn_ds_permute(4 * (here >> 4 == block ? here & 15 : 63), lane + 1);
        if (more) {
          const bool mine = (more >> lane) & 1;
          const int late = __builtin_amdgcn_ds_permute(4 * (mine ? after & 15 : 63), 64 + lane + 1);
          token = token ? token : late;
        }
      }
      write_block(p, turn, t0 - 1, token, (unsigned)block, kind, h0);
    }
  }

  static __device__ __forceinline__ void write_block(const PagedWriteParams& p, const Turn& turn, int64_t base,
                                                     int token, unsigned block, int kind, int h0) {
    const int lane = threadIdx.x & 63, lr = lane % LPR;
    const unsigned per_page = (unsigned)p.c.page_size / kPageRows;
    const unsigned page = block / per_page, within = block - page * per_page;
    const bool anew = __builtin_amdgcn_readlane(token, 0) != 0;
    int t[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) t[i] = __builtin_amdgcn_ds_bpermute(4 * (lane / LPR + i * RPI), token);
    const bool keys = ROPE && kind == 0;
    const Pieces<D, 8, INTER> pc(lr, turn.R);
    // (rows that stay as they are: 16 elements of a row side by side)
    const int first = keys ? pc.at[0] : 2 * lr, second = keys ? pc.at[1] : 2 * lr + 1;
    float c[NI][8], s[NI][8];
    if (keys) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (t[i]) pc.angles(turn, turn.pos ? turn.pos[base + t[i]] : (int)(base + t[i]), c[i], s[i]);
    }
    for (int h = h0; h < min(h0 + p.heads, p.c.Hkv); ++h) {
      const char* in = (kind ? p.v : p.k) + h * p.head_stride;
      char* out = (kind ? p.c.v : p.c.k) + (int64_t)page * p.c.page_stride + h * p.c.head_stride +
                  (int64_t)(within * kPageRows) * p.c.token_stride;
      uint8_t* scale = (kind ? p.c.vb : p.c.kb) + ((int64_t)page * p.c.Hkv + h) * per_page + within;
      int byte = 0;
      if (!anew) byte = *scale;
      i32x4 x[NI][2];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        x[i][0] = x[i][1] = i32x4{0, 0, 0, 0};
        if (t[i]) {
          const char* row = in + (base + t[i]) * p.token_stride;
          x[i][0] = *reinterpret_cast<const i32x4*>(row + first * 16);
          x[i][1] = *reinterpret_cast<const i32x4*>(row + second * 16);
        }
      }
      if (keys) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          float v[2][8];
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) unpack((uint32_t)x[i][n][k], v[n] + 2 * k);
          if (t[i]) pc.apply(v, c[i], s[i]);
#pragma unroll
          for (int n = 0; n < 2; ++n)    // the key as it would be stored without a cache
#pragma unroll
            for (int k = 0; k < 4; ++k) x[i][n][k] = pack(v[n] + 2 * k);
        }
      }
      // |bf16| compare as their bits; infinities and NaN, which do not count, are above all others
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          bits = max_u16x2(max_u16x2(bits, (uint32_t)x[i][0][k] & 0x7fff7fffu), (uint32_t)x[i][1][k] & 0x7fff7fffu);
      int most = wave_max((int)max(bits & 0xffffu, bits >> 16));
      const bool odd = most >= 0x7f80;
      if (odd) {
        bits = 0;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            bits = max_finite(max_finite(bits, (uint32_t)x[i][0][k]), (uint32_t)x[i][1][k]);
        most = wave_max((int)max(bits & 0xffffu, bits >> 16));
      }
      const int old = anew ? kScaleMin : min(max(__builtin_amdgcn_readfirstlane(byte) - 127, kScaleMin), kScaleMax);
      const int e = max(old, block_exponent((uint32_t)most));
      if (lane == 0) *scale = (uint8_t)(e + 127);

      i32x4 y[NI];
      if (odd || e == kScaleMax) {
        // (448 x 2^120 is no bf16 any more)
        const float inv = power_of_two(-e), limit = e == kScaleMax ? 240.f : 448.f;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t a = (uint32_t)x[i][k / 2][2 * (k % 2)], b = (uint32_t)x[i][k / 2][2 * (k % 2) + 1];
            y[i][k] = to_block4(bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b), inv, limit);
          }
      } else {
        // the instruction divides by the scale and rounds once, to nearest even (checked for every
        // bf16 and e); it does not saturate, and here nothing is above 448
        const float f = power_of_two(e);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t a = (uint32_t)x[i][k / 2][2 * (k % 2)], b = (uint32_t)x[i][k / 2][2 * (k % 2) + 1];
            s16x2 r = {0, 0};
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, a), f, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, b), f, true);
            y[i][k] = __builtin_bit_cast(int, r);
          }
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (!t[i]) continue;
        char* row = out + (lane / LPR + i * RPI) * p.c.token_stride;
        if (keys) {
          *reinterpret_cast<i32x2*>(row + first * 8) = i32x2{y[i][0], y[i][1]};
          *reinterpret_cast<i32x2*>(row + second * 8) = i32x2{y[i][2], y[i][3]};
        } else {
          *reinterpret_cast<i32x4*>(row + first * 8) = y[i];
        }
      }
      // a larger scale than the block had: its other rows
      if (!anew && e > old) {
        const float less = power_of_two(max(old - e, -100));
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if (t[i]) continue;
          i32x4* row = reinterpret_cast<i32x4*>(out + (lane / LPR + i * RPI) * p.c.token_stride + 16 * lr);
          i32x4 z = *row;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(z[k], false);
            const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(z[k], true);
            z[k] = to_block4(a[0], a[1], b[0], b[1], less, 448.f);
          }
          *row = z;
        }
      }
    }
  }
};

template <int D>
__global__ __launch_bounds__(256) void mala_paged_block_write_kernel(PagedWriteParams p) {
  BlockWriter<D, false, false>::run(p, Turn{}, blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

// Keys and values into a block-scaled cache by the first workgroups, queries by the others.
template <int D, bool INTER>
__global__ __launch_bounds__(256) void mala_paged_block_rope_kernel(PagedRopeWriteParams p) {
  if (blockIdx.x < p.kv_groups) {
    BlockWriter<D, true, INTER>::run(p.w, p.q.turn, blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  } else {
    const unsigned nx = (p.q.T + rope_tokens(D) - 1) / rope_tokens(D), i = blockIdx.x - p.kv_groups;
    turn_rows<D, false, false, INTER, false>(p.q, i % nx * rope_tokens(D), (int)(i / nx) * p.q.per);
  }
}

// The same for a cache of bf16, or of e4m3 with a scale per head: every row is its own.
template <int D, bool E4M3, bool INTER>
__global__ __launch_bounds__(256) void mala_paged_rope_write_kernel(PagedRopeWriteParams p) {
  constexpr int LPR = D / 16, TOK = rope_tokens(D);
  const unsigned nx = (p.q.T + TOK - 1) / TOK;
  if (blockIdx.x >= p.kv_groups) {
    const unsigned i = blockIdx.x - p.kv_groups;
    turn_rows<D, false, false, INTER, false>(p.q, i % nx * TOK, (int)(i / nx) * p.q.per);
    return;
  }
  const PagedWriteParams& w = p.w;
  const Turn& turn = p.q.turn;
  const unsigned t = blockIdx.x % nx * TOK + threadIdx.x / LPR, P = w.c.page_size;
  if (t >= p.q.T) return;
  const int slot = w.slots[t], lr = threadIdx.x % LPR;
  if (slot < 0 || (unsigned)slot >= w.c.num_pages * P) return;
  const unsigned page = slot / P, row = slot - page * P;
  const int kind = blockIdx.x / nx % 2, h0 = blockIdx.x / nx / 2 * w.heads;
  const Pieces<D, 8, INTER> pc(lr, turn.R);
  float c[8], s[8];
  if (!kind) pc.angles(turn, turn.pos ? turn.pos[t] : (int)t, c, s);
  for (int h = h0; h < min(h0 + w.heads, w.c.Hkv); ++h) {
    const char* x = (kind ? w.v : w.k) + t * w.token_stride + h * w.head_stride;
    char* out = (kind ? w.c.v : w.c.k) + page * w.c.page_stride + h * w.c.head_stride + row * w.c.token_stride;
    float v[2][8];
    load_piece<false>(x + pc.at[0] * 16, v[0]);
    load_piece<false>(x + pc.at[1] * 16, v[1]);
    if (!kind) pc.apply(v, c, s);
    const float* scales = kind ? w.c.vs : w.c.ks;
    const float scale = E4M3 && scales ? scales[h] : 1.f;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      i32x4 y;                           // (a value as it is, a rotated key rounded)
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = pack(v[n] + 2 * k);
      if constexpr (E4M3) {
        int e[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t a = (uint32_t)y[2 * i], b = (uint32_t)y[2 * i + 1];
          e[i] = to_e4m3x4(bf16_lo(a) / scale, bf16_hi(a) / scale, bf16_lo(b) / scale, bf16_hi(b) / scale);
        }
        *reinterpret_cast<i32x2*>(out + pc.at[n] * 8) = i32x2{e[0], e[1]};
      } else {
        *reinterpret_cast<i32x4*>(out + pc.at[n] * 16) = y;
      }
    }
  }
}

}  // namespace

// Workgroups (of four wavefronts) of the keys and values
static unsigned block_write_groups(PagedWriteParams& p, bool rope) {
  const BlockWritePlan x = block_write_plan(p.T, p.c.Hkv, rope);
  p.chunk = x.chunk;
  p.heads = x.heads;
  return (unsigned)((x.waves + 3) / 4);
}

hipError_t launch_paged_block_write(PagedWriteParams p, int D, hipStream_t st) {
  const dim3 grid(block_write_groups(p, false));
  if (D == 128)
    hipLaunchKernelGGL(mala_paged_block_write_kernel<128>, grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(mala_paged_block_write_kernel<64>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

template <int D, bool INTER>
static void launch_rope_write_t(PagedRopeWriteParams& p, hipStream_t st) {
  const unsigned nx = (p.q.T + rope_tokens(D) - 1) / rope_tokens(D);
  unsigned q_groups = 0;
  if (p.q.r[0].H) {
    p.q.per = rope_heads_per_group(p.q.T, p.q.r[0].H, D);
    q_groups = nx * ((p.q.r[0].H + p.q.per - 1) / p.q.per);
  }
  if (p.w.c.fmt == kCacheBlock) {
    p.kv_groups = block_write_groups(p.w, true);
  } else {
    p.w.heads = rope_heads_per_group(p.w.T, p.w.c.Hkv, D);
    p.kv_groups = nx * 2 * ((p.w.c.Hkv + p.w.heads - 1) / p.w.heads);
  }
  const dim3 grid(p.kv_groups + q_groups);
  if (p.w.c.fmt == kCacheBlock)
    hipLaunchKernelGGL((mala_paged_block_rope_kernel<D, INTER>), grid, dim3(256), 0, st, p);
  else if (p.w.c.fmt == kCacheE4M3)
    hipLaunchKernelGGL((mala_paged_rope_write_kernel<D, true, INTER>), grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((mala_paged_rope_write_kernel<D, false, INTER>), grid, dim3(256), 0, st, p);
}
template <int D>
static void launch_rope_write_d(PagedRopeWriteParams& p, hipStream_t st) {
  p.q.turn.interleaved ? launch_rope_write_t<D, true>(p, st) : launch_rope_write_t<D, false>(p, st);
}

hipError_t launch_paged_rope_write(PagedRopeWriteParams p, int D, hipStream_t st) {
  D == 128 ? launch_rope_write_d<128>(p, st) : launch_rope_write_d<64>(p, st);
  return hipGetLastError();
}

}  // namespace mala
