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
  bool heads_first;        // order of the workgroups
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
// pi / 4 are their Taylor sums: the first terms left out are x^11 / 11! (2^-29 at pi / 4, a 32nd of half a
// step of 1) and x^12 / 12! (2^-33); with all roundings the sums are within 0.9 x 2^-24 of sin and cos.
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

// The 16 elements of a row that a lane owns (D / 16 lanes a row): pieces of E elements, so that each
// is loaded and stored at once and neighbouring lanes' pieces lie side by side.  Pieces 2 i and 2 i + 1
// hold both elements of E pairs (half), or each piece E / 2 pairs (interleaved: INTER).
template <int D, int E, bool INTER>
struct Pieces {
  static constexpr int LPR = D / 16, N = 16 / E, HALF = D / (2 * E);
  int at[N];             // their numbers in the row
  bool turned[N];

  __device__ __forceinline__ Pieces(int lane_of_row, int R) {
    const int pairs = R / (2 * E);       // pieces that hold first elements (half)
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const int n = i * LPR + lane_of_row;
      if constexpr (INTER) {
        at[2 * i] = n;
        at[2 * i + 1] = n + HALF;
        turned[2 * i] = n * E < R;
        turned[2 * i + 1] = (n + HALF) * E < R;
      } else {
        turned[2 * i] = turned[2 * i + 1] = n < pairs;
        at[2 * i] = n < pairs ? n : n + pairs;
        at[2 * i + 1] = n < pairs ? n + pairs : n + HALF;
      }
    }
  }
  // Pairs that piece n is the (first) piece of, and the number of the first of them.
  static constexpr int pairs_of(int n) { return INTER ? E / 2 : n % 2 ? 0 : E; }
  __device__ __forceinline__ int first_pair(int n) const { return at[n] * (INTER ? E / 2 : E); }

  // cos and sin of the lane's eight pairs, as far as they are turned
  __device__ __forceinline__ void angles(const Turn& turn, int pos, float (&c)[8], float (&s)[8]) const {
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (turned[n])
#pragma unroll
        for (int k = 0; k < pairs_of(n); ++k)
          turn_of(pos, turn.inv_freq[first_pair(n) + k], turn.scale, turn.sin_scale, c[n * (E / 2) + k],
                  s[n * (E / 2) + k]);
  }
  __device__ __forceinline__ void apply(float (&x)[N][E], const float (&c)[8], const float (&s)[8]) const {
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (turned[n])
#pragma unroll
        for (int k = 0; k < pairs_of(n); ++k) {
          const int slot = n * (E / 2) + k;
          if constexpr (INTER)
            turn_pair(x[n][2 * k], x[n][2 * k + 1], c[slot], s[slot]);
          else
            turn_pair(x[n][k], x[n + 1][k], c[slot], s[slot]);
        }
  }
};

__device__ __forceinline__ void unpack(uint32_t u, float* x) {
  x[0] = __uint_as_float(u << 16);
  x[1] = __uint_as_float(u & 0xffff0000u);
}
__device__ __forceinline__ int pack(const float* x) {
  return __builtin_bit_cast(int, __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2));
}

// A piece of E elements as it lies in memory, bf16 or fp32: 8, 16 or 32 bytes.
template <bool F32, int E>
struct RawPiece {
  static constexpr int WORDS = E * (F32 ? 4 : 2) / 4;
  int d[WORDS];

  // ONCE: past the caches
  template <bool ONCE>
  __device__ __forceinline__ void load(const char* p) {
    typedef int vec __attribute__((ext_vector_type(WORDS < 4 ? WORDS : 4)));
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      const vec* at = reinterpret_cast<const vec*>(p + 4 * i);
      const vec x = ONCE ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
      for (int k = 0; k < 4 && k < WORDS; ++k) d[i + k] = x[k];
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    typedef int vec __attribute__((ext_vector_type(WORDS < 4 ? WORDS : 4)));
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      vec x;
#pragma unroll
      for (int k = 0; k < 4 && k < WORDS; ++k) x[k] = d[i + k];
      __builtin_nontemporal_store(x, reinterpret_cast<vec*>(p + 4 * i));
    }
  }
  __device__ __forceinline__ void get(float (&x)[E]) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (F32)
        x[i] = __int_as_float(d[i]);
      else
        unpack((uint32_t)d[i], x + 2 * i);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (F32)
        d[i] = __float_as_int(x[i]);
      else
        d[i] = pack(x + 2 * i);
    }
  }
};
// Exchanges a with lane `with`'s b where `first`, b with its a where not; with itself: nothing.
template <class Raw>
__device__ __forceinline__ void swap_pieces(Raw& a, Raw& b, int with, bool first) {
#pragma unroll
  for (int i = 0; i < Raw::WORDS; ++i) {
    const int got = __builtin_amdgcn_ds_bpermute(4 * with, first ? b.d[i] : a.d[i]);
    (first ? b.d[i] : a.d[i]) = got;
  }
}

// Rows of the heads [h0, h0 + per) of 256 / (D / 16) tokens from number `first` on (of all
// batches'), by a workgroup of 256 threads: D / 16 lanes a row, a thread keeps its token and with
// it the angles.  ONCE: x is loaded past the caches.  HEADS: heads whose rows are loaded at a time.  (In
// place: a row is read by the lanes that write it, before they do.)
template <int D, bool IN32, bool OUT32, bool INTER, bool ONCE, int HEADS>
__device__ __forceinline__ void turn_rows(const RopeParams& p, unsigned first, int h0) {
  // (whole pieces at a store: half lines stored at a time cost more than half lines loaded: 16000
  // tokens' gradients, fp32 to bf16, 86 us in pieces of 8, 89 of 4)
  constexpr int LPR = D / 16, E = OUT32 ? 4 : 8, N = 16 / E;
  constexpr int IN = E * (IN32 ? 4 : 2), OUT = E * (OUT32 ? 4 : 2);     // bytes of a piece
  const unsigned i = first + threadIdx.x / LPR;
  if (i >= p.B * p.T) return;
  const unsigned b = i / p.T, t = i - b * p.T;
  const Pieces<D, E, INTER> pc(threadIdx.x % LPR, p.turn.R);
  float c[8], s[8];
  pc.angles(p.turn, p.turn.pos ? p.turn.pos[b * p.turn.pos_b + t] : (int)t, c, s);
  // Where up to half of each head turns, the two halves of a turned pair come from one line: lanes then
  // load and store pieces lane and lane + LPR, whole lines, and swap one of them for the one they turn.
  const bool lines = !INTER && E == 8 && 2 * p.turn.R <= D;
  const int lr = threadIdx.x % LPR, lane = threadIdx.x & 63, half = p.turn.R / 16;
  const bool low = lr < half;
  const int with = low ? lane + half : lr < 2 * half ? lane - half : lane;
  int at[N];
#pragma unroll
  for (int n = 0; n < N; ++n) at[n] = lines ? lr + n * LPR : pc.at[n];
  const int heads = p.r[0].H + p.r[1].H, h1 = min(h0 + p.per, heads);
  const auto of = [&](int h, auto RopeRows::* f) { return h >= p.r[0].H ? p.r[1].*f : p.r[0].*f; };
  for (int h = h0; h < h1; h += HEADS) {
    RawPiece<IN32, E> in[HEADS][N];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
      const int g = min(h + k, h1 - 1), hr = g >= p.r[0].H ? g - p.r[0].H : g;
      const char* x = of(g, &RopeRows::x) + hr * of(g, &RopeRows::xh) +
                      (b * of(g, &RopeRows::xb) + t * of(g, &RopeRows::xt));
#pragma unroll
      for (int n = 0; n < N; ++n) in[k][n].template load<ONCE>(x + at[n] * IN);
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
      const int g = h + k, hr = g >= p.r[0].H ? g - p.r[0].H : g;
      if (g >= h1) break;
      RawPiece<OUT32, E> y[N];
      float v[N][E];
      if (lines) swap_pieces(in[k][0], in[k][1], with, low);
#pragma unroll
      for (int n = 0; n < N; ++n) in[k][n].get(v[n]);
      pc.apply(v, c, s);
#pragma unroll
      for (int n = 0; n < N; ++n) y[n].set(v[n]);
      if (lines) swap_pieces(y[0], y[1], with, low);
      char* out = of(g, &RopeRows::out) + hr * of(g, &RopeRows::oh) +
                  (b * of(g, &RopeRows::ob) + t * of(g, &RopeRows::ot));
#pragma unroll
      for (int n = 0; n < N; ++n) y[n].store(out + at[n] * OUT);
    }
  }
}

hipError_t launch_rope(RopeParams p, int D, bool in32, bool out32, hipStream_t st);
hipError_t launch_paged_rope_write(PagedRopeWriteParams p, int D, hipStream_t st);

}  // namespace mala
