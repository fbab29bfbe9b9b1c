// Rotary positions: parameter blocks, launchers, and the device code that the rotation and the
// rotated cache write share (both give the same bits).
//
// Pair i < R / 2 of a row at position n turns by theta = n inv_freq[i]:
//   (a, b) -> scale (a cos - b sin, b cos + a sin)
// half: elements i and i + R / 2; interleaved: 2 i and 2 i + 1.  Elements from R on stay.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mala_device.h"
#include "mala_paged.h"

namespace mala {

// Rows of one tensor: token t, head h of batch b at byte b * xb + h * xh + t * xt of x (out alike).
struct RopeRows {
  const char* x;
  char* out;
  int64_t xb, xh, xt, ob, oh, ot;
  int H;
};

struct Turn {
  const int32_t* pos;      // [B][T] (batches pos_b elements apart), or null: position t
  int64_t pos_b;
  const double* inv_freq;  // [R / 2]
  int R, interleaved;      // R: a multiple of 16
  float scale, sin_scale;  // sin_scale: -scale for the transposed rotation
};

struct RopeParams {
  RopeRows r[2];           // r[1].H = 0: one tensor
  Turn turn;
  unsigned B, T;
  int per;                 // heads per workgroup
};

struct PagedRopeWriteParams {
  PagedWriteParams w;
  RopeParams q;            // B = 1, T tokens; H = 0: no queries; turn: for the keys too
  unsigned kv_groups;      // workgroups of the keys and values, the queries' follow
};

// cos and sin of pos inv_freq, each times its scale.
//
// The angle in quarter turns is pos (2 / pi) inv_freq, of which only the distance to the nearest
// whole number counts: as fp32 it would lose log2(pos) bits.  Both products are taken to twice 53
// bits (a product and its exact remainder), so that what is left of a quarter turn is right to
// 2^-53 of the quarter turn at any position, and then rounded to fp32 once.  sin and cos of up to
// pi / 4 are their Taylor sums (the terms left out are below 2^-32).
__device__ __forceinline__ void turn_of(int pos, double inv_freq, float scale, float sin_scale,
                                        float& c, float& s) {
#pragma clang fp contract(off)
  constexpr double kHi = 0x1.45f306dc9c883p-1, kLo = -0x1.6b01ec5417056p-55;   // 2 / pi
  constexpr double kHalfPi = 0x1.921fb54442d18p+0;
  const double n = pos, fh = inv_freq * kHi;
  const double fl = __builtin_fma(inv_freq, kHi, -fh) + inv_freq * kLo;
  const double t = n * fh, rest = __builtin_fma(n, fh, -t) + n * fl;
  const double whole = __builtin_rint(t);
  const float x = (float)(((t - whole) + rest) * kHalfPi);
  const int quadrant = (int)(__builtin_amdgcn_fract(whole * 0.25) * 4.0);
  const float z = x * x;
  float a = 0x1.71de3ap-19f;                          // 1 / 9!
  a = __builtin_fmaf(a, z, -0x1.a01a02p-13f);         // 1 / 7!
  a = __builtin_fmaf(a, z, 0x1.111112p-7f);           // 1 / 5!
  a = __builtin_fmaf(a, z, -0x1.555556p-3f);          // 1 / 3!
  const float sine = __builtin_fmaf(a * z, x, x);
  float b = -0x1.27e4fcp-22f;                         // 1 / 10!
  b = __builtin_fmaf(b, z, 0x1.a01a02p-16f);          // 1 / 8!
  b = __builtin_fmaf(b, z, -0x1.6c16c2p-10f);         // 1 / 6!
  b = __builtin_fmaf(b, z, 0x1.555556p-5f);           // 1 / 4!
  b = __builtin_fmaf(b, z, -0.5f);
  const float cosine = __builtin_fmaf(b, z, 1.f);
  const bool swap = quadrant & 1;
  const float cq = swap ? sine : cosine, sq = swap ? cosine : sine;
  c = ((quadrant + 1) & 2 ? -cq : cq) * scale;
  s = (quadrant & 2 ? -sq : sq) * sin_scale;
}

// The rotation of a pair; one product rounded, the other fused.
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float bs = b * s, as = a * s, a0 = a;
  a = __builtin_fmaf(a0, c, -bs);
  b = __builtin_fmaf(b, c, as);
}

// A lane owns 16 elements of a row, two pieces of 8 which hold both elements of 8 pairs: pairs
// 8 piece .. + 7 where the lane's number is below R / 16.
struct Pieces {
  int first, second;     // numbers of the two pieces
  bool turned;
};
__device__ __forceinline__ Pieces pieces_of(int lane_of_row, int R, int interleaved) {
  Pieces x = {2 * lane_of_row, 2 * lane_of_row + 1, 16 * lane_of_row < R};
  if (x.turned && !interleaved) {
    x.first = lane_of_row;
    x.second = lane_of_row + R / 16;
  }
  return x;
}
// x: the two pieces' elements, in order; c, s of the lane's 8 pairs
__device__ __forceinline__ void turn_pieces(float (&x)[16], const float (&c)[8], const float (&s)[8],
                                            int interleaved) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (interleaved)
      turn_pair(x[2 * i], x[2 * i + 1], c[i], s[i]);
    else
      turn_pair(x[i], x[8 + i], c[i], s[i]);
  }
}

// Eight elements at p, bf16 or fp32.
template <bool F32>
__device__ __forceinline__ void load_piece(const char* p, float* x) {
  if constexpr (F32) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  } else {
    const i32x4 a = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float((uint32_t)a[i] << 16);
      x[2 * i + 1] = __uint_as_float((uint32_t)a[i] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ i32x4 to_bf16x8(const float* x) {
  i32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    y[i] = __builtin_bit_cast(int, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
  return y;
}
template <bool F32>
__device__ __forceinline__ void store_piece(char* p, const float* x) {
  if constexpr (F32) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 16) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    *reinterpret_cast<i32x4*>(p) = to_bf16x8(x);
  }
}

// Rows of the heads [h0, h0 + per) of 256 / (D / 16) tokens from number `first` on (of all
// batches'), by a workgroup of 256 threads: D / 16 lanes a row, a thread keeps its token and with
// it the angles.
template <int D, bool IN32, bool OUT32>
__device__ __forceinline__ void turn_rows(const RopeParams& p, unsigned first, int h0) {
  constexpr int LPR = D / 16, IN = IN32 ? 4 : 2, OUT = OUT32 ? 4 : 2;
  const unsigned i = first + threadIdx.x / LPR;
  if (i >= p.B * p.T) return;
  const int lr = threadIdx.x % LPR;
  const unsigned b = i / p.T, t = i - b * p.T;
  const Pieces pc = pieces_of(lr, p.turn.R, p.turn.interleaved);
  float c[8], s[8];
  if (pc.turned) {
    const int pos = p.turn.pos ? p.turn.pos[b * p.turn.pos_b + t] : (int)t;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      turn_of(pos, p.turn.inv_freq[8 * lr + k], p.turn.scale, p.turn.sin_scale, c[k], s[k]);
  }
  const int heads = p.r[0].H + p.r[1].H, h1 = min(h0 + p.per, heads);
  for (int h = h0; h < h1; ++h) {
    const RopeRows& r = p.r[h >= p.r[0].H];
    const int hr = h >= p.r[0].H ? h - p.r[0].H : h;
    const char* x = r.x + b * r.xb + hr * r.xh + t * r.xt;
    char* out = r.out + b * r.ob + hr * r.oh + t * r.ot;
    float v[16];
    load_piece<IN32>(x + pc.first * 8 * IN, v);
    load_piece<IN32>(x + pc.second * 8 * IN, v + 8);
    if (pc.turned) turn_pieces(v, c, s, p.turn.interleaved);
    store_piece<OUT32>(out + pc.first * 8 * OUT, v);
    store_piece<OUT32>(out + pc.second * 8 * OUT, v + 8);
  }
}

hipError_t launch_rope(RopeParams p, int D, bool in32, bool out32, hipStream_t st);
hipError_t launch_paged_rope_write(PagedRopeWriteParams p, int D, hipStream_t st);

}  // namespace mala
