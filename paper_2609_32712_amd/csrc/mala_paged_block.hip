// Rows into pages of e4m3 values with a scale per block of 16 rows and KV head, and the rotation of
// a step's queries and keys in the same launch (gfx950).
//
// A block's scale is 2^e.  e of new rows is the least integer with amax <= 448 2^e (finite values
// alone), kept in [kScaleMin, kScaleMax]; a block whose row 0 is new starts anew, any other one
// takes the larger of its e and the new one, and when that grows its other rows are rounded again,
// to nearest even as the new ones.  Scales are powers of two so that this second rounding is exact
// but where a value leaves the normal range, and so that value x scale is a bf16.
//
// What bounds it: HBM (2 bytes read and 1 written per value): 20000 tokens of 8 heads 20 us, 5.8 TB/s;
// 16000 turned ones with 32 heads' queries 67 us, 5.4 TB/s; small calls the chain slots -> scale ->
// stores (64 decodes 3.5 us, turned and with their queries 4.3).
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

// Keys and values of the blocks whose first token (of this call) is among the workgroup's chunk of
// tokens.  Every wavefront finds the rows of those blocks by itself, from the slots around the
// tokens, by ballots and lane exchanges; D / 16 lanes take a row.
//   - a block with several tokens (prompts): one head of K or of V at a time to a wavefront, its
//     rows over the lanes;
//   - tokens that are their block's only one (decodes): a token and head of K or of V to each D / 16
//     lanes.  (As blocks, whose instructions serve 16 rows: 1000 tokens of 8 heads 9.1 us.)
// The angles of a token serve all its heads: the workgroup computes them once.
template <int D, bool ROPE, bool INTER>
struct BlockWriter {
  static constexpr int LPR = D / 16, RPI = 64 / LPR, NI = kPageRows / RPI;   // rows at a time, times
  static constexpr int ROW = D / 2 + 2;    // (a row's angles 16 bytes off the next one's banks)
  static_assert(kBlockChunk <= kPageRows, "a table of angles for a block's rows or a chunk's tokens");
  // One table is read while the next one is written.
  struct Turns {
    __attribute__((aligned(16))) f32x2 at[ROPE ? 2 : 1][ROPE ? kPageRows * ROW : 1];
  };
  // A block of one head, as it comes in
  struct Rows {
    i32x4 x[NI][2];
    int byte;
  };

  const PagedWriteParams& p;
  const Turn& turn;
  const int lane, w, lr;
  const unsigned per_page;                 // blocks of a page
  const Pieces<D, 8, INTER> pc;
  int64_t base = 0;                        // tokens are counted from here, + 1 so that 0 is none
  // the block: its place, and the tokens of this lane's rows
  unsigned within = 0, page = 0;
  int t[NI];
  bool anew = false;
  int pos_here = 0, pos_after = 0;         // positions of the 64 tokens from t0 on, and of the next

  __device__ __forceinline__ BlockWriter(const PagedWriteParams& p, const Turn& turn)
      : p(p), turn(turn), lane(threadIdx.x & 63), w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)),
        lr(threadIdx.x % LPR), per_page((unsigned)p.c.page_size / kPageRows), pc(threadIdx.x % LPR, turn.R) {}

  __device__ __forceinline__ void run(unsigned group, Turns& turns) {
    const int parts = block_write_parts(p.c.Hkv, p.units);
    const unsigned chunk = group / parts, part = group - chunk * parts;
    const int u_lo = (int)part * 4 * p.units, u_hi = min(u_lo + 4 * p.units, 2 * p.c.Hkv);
    const int64_t t0 = (int64_t)chunk * p.chunk;
    base = t0 - 1;
    const int slots = (int)(p.c.num_pages * (unsigned)p.c.page_size);
    const auto load_slot = [&](int64_t n) { return n >= 0 && n < p.T ? p.slots[n] : -1; };
    const auto in_pool = [&](int s) { return s < slots && s >= 0 ? s : -1; };
    // The slots of the tokens around, and their positions.  A chunk of one token, most likely alone: its
    // rows and angles are fetched beside the slots.
    int before = load_slot(t0 - 64 + lane), here = load_slot(t0 + lane), after = -1;
    if constexpr (ROPE) pos_here = pos_of(t0 + lane);
    i32x4 early[2];
    if (p.chunk == 1) {
      load_one(1, min(u_lo + w * RPI + lane / LPR, u_hi - 1), early);
      if constexpr (ROPE) table(turns.at[0], 1, 1);
    } else {
      after = load_slot(t0 + 64 + lane);
      if constexpr (ROPE) pos_after = pos_of(t0 + 64 + lane);
    }
    before = in_pool(before);
    here = in_pool(here);
    after = in_pool(after);
    uint64_t todo = __builtin_amdgcn_ballot_w64(here >= 0 && lane < p.chunk), ones = 0;
    int tables = 0;
    while (todo) {                        // (the same for the workgroup's wavefronts)
      const int ci = __builtin_ctzll(todo), block = __builtin_amdgcn_readlane(here, ci) >> 4;
      // (-1 >> 4 is no block's number.  Tokens of a block lie within 64: those before from lane ci + 1 on,
      // those after below lane ci)
      const uint64_t same = __builtin_amdgcn_ballot_w64(here >> 4 == block);
      todo &= ~same;
      if (__builtin_amdgcn_ballot_w64(before >> 4 == block) >> ci >> 1) continue;
      const uint64_t more =
          p.chunk > 1 ? __builtin_amdgcn_ballot_w64(after >> 4 == block) & ((1ull << ci) - 1) : 0;
      if (!(same & (same - 1)) && !more) {
        ones |= same;
        continue;
      }
      // token of row r of the block in lane r < 16; 0 for none (of tokens with the same slot, one's
      // number arrives)
      int token = __builtin_amdgcn_ds_permute(4 * (here >> 4 == block ? here & 15 : 63), lane + 1);
      if (more) {
        const bool mine = (more >> lane) & 1;
        const int late = __builtin_amdgcn_ds_permute(4 * (mine ? after & 15 : 63), 64 + lane + 1);
        token = token ? token : late;
      }
      page = (unsigned)block / per_page;
      within = (unsigned)block - page * per_page;
      anew = __builtin_amdgcn_readlane(token, 0) != 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) t[i] = __builtin_amdgcn_ds_bpermute(4 * (lane / LPR + i * RPI), token);

      Rows now, next;
      if (u_lo + w < u_hi) load(u_lo + w, now);      // on its way while the angles are computed
      const f32x2* angles = nullptr;
      if constexpr (ROPE) {
        f32x2* to = turns.at[++tables & 1];
        table(to, token, kPageRows);
        __syncthreads();
        angles = to;
      }
      for (int u = u_lo + w; u < u_hi; u += 4) {
        if (u + 4 < u_hi) load(u + 4, next);
        write(u, now, angles);
        now = next;
      }
    }
    if (!ones) return;
    // tokens that are alone, in lanes 0, 1, .. (lanes behind the last one are not asked)
    const int count = __builtin_popcountll(ones);
    const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(ones >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)ones, 0));
    const int token = __builtin_amdgcn_ds_permute(4 * ((ones >> lane) & 1 ? rank : 63), lane + 1);
    const f32x2* angles = turns.at[0];
    if constexpr (ROPE) {
      if (p.chunk > 1) {
        f32x2* to = turns.at[++tables & 1];
        table(to, lane < count ? token : 0, count);
        angles = to;
      }
      __syncthreads();
    }
    const int per_token = u_hi - u_lo;
    for (int i0 = w * RPI; i0 < count * per_token; i0 += 4 * RPI) {
      const int i = min(i0 + lane / LPR, count * per_token - 1), j = i / per_token, u = u_lo + i - j * per_token;
      const int n = __builtin_amdgcn_ds_bpermute(4 * j, token);
      const int slot = __builtin_amdgcn_ds_bpermute(4 * (n - 1), here);
      if (p.chunk > 1 || i0 != w * RPI) load_one(n, u, early);
      if (i0 + lane / LPR < count * per_token) write_one(u, slot, early, angles + j * ROW);
    }
  }

  // Unit u of the workgroup's 2 Hkv: a head of K, or behind those of V.
  __device__ __forceinline__ int kind_of(int u) const { return u >= p.c.Hkv; }
  __device__ __forceinline__ int head_of(int u) const { return u >= p.c.Hkv ? u - p.c.Hkv : u; }
  __device__ __forceinline__ uint8_t* scale_of(int u, unsigned page, unsigned within) const {
    return (kind_of(u) ? p.c.vb : p.c.kb) + ((int64_t)page * p.c.Hkv + head_of(u)) * per_page + within;
  }
  __device__ __forceinline__ char* block_of(int u, unsigned page, unsigned within) const {
    return (kind_of(u) ? p.c.v : p.c.k) + (int64_t)page * p.c.page_stride + head_of(u) * p.c.head_stride +
           (int64_t)(within * kPageRows) * p.c.token_stride;
  }
  __device__ __forceinline__ const char* row_of(int u, int token) const {
    return (kind_of(u) ? p.v : p.k) + head_of(u) * p.head_stride + (base + token) * p.token_stride;
  }
  // (rows that stay as they are: 16 elements of a row side by side)
  __device__ __forceinline__ int piece(int u, int n) const { return ROPE && !kind_of(u) ? pc.at[n] : 2 * lr + n; }

  __device__ __forceinline__ int pos_of(int64_t n) const {
    return n >= p.T ? 0 : turn.pos ? turn.pos[n] : (int)n;
  }
  // cos and sin of the first `rows` tokens of lanes 0, 1, .., by the workgroup.  (Lanes are asked by all
  // lanes: one that is switched off would answer 0.)
  __device__ __forceinline__ void table(f32x2* to, int token, int rows) const {
    const int pairs = turn.R / 2, own = 4 * ((token - 1) & 63);
    const int near = __builtin_amdgcn_ds_bpermute(own, pos_here), far = __builtin_amdgcn_ds_bpermute(own, pos_after);
    const int own_pos = token > 64 ? far : near;
    for (int i0 = 0; i0 < rows * pairs; i0 += 256) {
      const int i = i0 + (int)threadIdx.x, row = min(i / pairs, rows - 1), pair = i - row * pairs;
      const int n = __builtin_amdgcn_ds_bpermute(4 * row, token), pos = __builtin_amdgcn_ds_bpermute(4 * row, own_pos);
      if (!n || i >= rows * pairs) continue;
      float c, s;
      turn_of(pos, turn.inv_freq[pair], turn.scale, turn.sin_scale, c, s);
      to[row * ROW + pair] = f32x2{c, s};
    }
  }

  // A row's two pieces turned, and rounded to bf16: the key as it would be stored without a cache.
  __device__ __forceinline__ void turn_row(i32x4 (&x)[2], const f32x2* angles) const {
    float v[2][8], c[8], s[8];
#pragma unroll
    for (int n = 0; n < 2; ++n)
      if (pc.turned[n]) {
        const f32x2* from = angles + pc.first_pair(n);
#pragma unroll
        for (int k = 0; k < pc.pairs_of(n); ++k) {
          c[4 * n + k] = from[k][0];
          s[4 * n + k] = from[k][1];
        }
      }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int k = 0; k < 4; ++k) unpack((uint32_t)x[n][k], v[n] + 2 * k);
    pc.apply(v, c, s);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[n][k] = pack(v[n] + 2 * k);
  }
  // |bf16| compare as their bits; infinities and NaN, which do not count, are above all others.
  static __device__ __forceinline__ uint32_t largest(const i32x4 (&x)[2], uint32_t bits) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      bits = max_u16x2(max_u16x2(bits, (uint32_t)x[0][k] & 0x7fff7fffu), (uint32_t)x[1][k] & 0x7fff7fffu);
    return bits;
  }
  static __device__ __forceinline__ uint32_t largest_finite(const i32x4 (&x)[2], uint32_t bits) {
#pragma unroll
    for (int k = 0; k < 4; ++k) bits = max_finite(max_finite(bits, (uint32_t)x[0][k]), (uint32_t)x[1][k]);
    return bits;
  }
  // e4m3 bytes of two pieces over 2^e.  The instruction divides by the scale and rounds once, to nearest
  // even (checked for every bf16 and e); it does not saturate: where something may be above 448, or
  // above 240 for the largest e (448 x 2^120 is no bf16 any more), the values are limited first.
  static __device__ __forceinline__ i32x4 over_scale(const i32x4 (&x)[2], int e) {
    const float f = power_of_two(e);
    i32x4 y;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = (uint32_t)x[k / 2][2 * (k % 2)], b = (uint32_t)x[k / 2][2 * (k % 2) + 1];
      s16x2 r = {0, 0};
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, a), f, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, b), f, true);
      y[k] = __builtin_bit_cast(int, r);
    }
    return y;
  }
  static __device__ __forceinline__ i32x4 over_scale_limited(const i32x4 (&x)[2], int e) {
    const float inv = power_of_two(-e), limit = e == kScaleMax ? 240.f : 448.f;
    i32x4 y;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = (uint32_t)x[k / 2][2 * (k % 2)], b = (uint32_t)x[k / 2][2 * (k % 2) + 1];
      y[k] = to_block4(bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b), inv, limit);
    }
    return y;
  }
  static __device__ __forceinline__ int held_exponent(int byte) {
    return min(max(byte - 127, kScaleMin), kScaleMax);
  }
  // A row of a block under a larger scale: rounded again
  static __device__ __forceinline__ void rescale(char* at, int grown) {
    const float less = power_of_two(max(-grown, -100));
    i32x4* row = reinterpret_cast<i32x4*>(at);
    i32x4 z = *row;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(z[k], false);
      const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(z[k], true);
      z[k] = to_block4(a[0], a[1], b[0], b[1], less, 448.f);
    }
    *row = z;
  }
  __device__ __forceinline__ void store_row(char* row, bool keys, i32x4 y) const {
    if (keys) {
      __builtin_nontemporal_store((i32x2{y[0], y[1]}), reinterpret_cast<i32x2*>(row + pc.at[0] * 8));
      __builtin_nontemporal_store((i32x2{y[2], y[3]}), reinterpret_cast<i32x2*>(row + pc.at[1] * 8));
    } else {
      __builtin_nontemporal_store(y, reinterpret_cast<i32x4*>(row + 16 * lr));
    }
  }

  // ------------------------------------------------------------ a block of several tokens
  __device__ __forceinline__ void load(int u, Rows& to) const {
    to.byte = 0;
    if (!anew) to.byte = *scale_of(u, page, within);
    const int first = piece(u, 0), second = piece(u, 1);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      to.x[i][0] = to.x[i][1] = i32x4{0, 0, 0, 0};
      if (t[i]) {
        const char* row = row_of(u, t[i]);
        to.x[i][0] = *reinterpret_cast<const i32x4*>(row + first * 16);
        to.x[i][1] = *reinterpret_cast<const i32x4*>(row + second * 16);
      }
    }
  }
  __device__ __forceinline__ void write(int u, Rows& rows, const f32x2* angles) const {
    const bool keys = ROPE && !kind_of(u);
    auto& x = rows.x;
    if (keys) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (t[i]) turn_row(x[i], angles + (lane / LPR + i * RPI) * ROW);
    }
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) bits = largest(x[i], bits);
    int most = wave_max((int)max(bits & 0xffffu, bits >> 16));
    const bool odd = most >= 0x7f80;
    if (odd) {
      bits = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) bits = largest_finite(x[i], bits);
      most = wave_max((int)max(bits & 0xffffu, bits >> 16));
    }
    const int old = anew ? kScaleMin : held_exponent(__builtin_amdgcn_readfirstlane(rows.byte));
    const int e = max(old, block_exponent((uint32_t)most));
    if (lane == 0) *scale_of(u, page, within) = (uint8_t)(e + 127);
    i32x4 y[NI];
    if (odd || e == kScaleMax) {
#pragma unroll
      for (int i = 0; i < NI; ++i) y[i] = over_scale_limited(x[i], e);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) y[i] = over_scale(x[i], e);
    }
    char* out = block_of(u, page, within);
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (t[i]) store_row(out + (lane / LPR + i * RPI) * p.c.token_stride, keys, y[i]);
    if (!anew && e > old) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (!t[i]) rescale(out + (lane / LPR + i * RPI) * p.c.token_stride + 16 * lr, e - old);
    }
  }

  // ------------------------------------------------------------ a token alone, D / 16 lanes
  __device__ __forceinline__ void load_one(int token, int u, i32x4 (&x)[2]) const {
    const char* row = row_of(u, token);
    x[0] = *reinterpret_cast<const i32x4*>(row + piece(u, 0) * 16);
    x[1] = *reinterpret_cast<const i32x4*>(row + piece(u, 1) * 16);
  }
  // the largest of the row's lanes
  static __device__ __forceinline__ int row_max(uint32_t bits) {
    int x = (int)max(bits & 0xffffu, bits >> 16);
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true));     // quad_perm: lane ^ 1
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true));     // quad_perm: lane ^ 2
    if constexpr (LPR == 8)
      x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true));  // row_half_mirror
    return x;
  }
  __device__ __forceinline__ void write_one(int u, int slot, i32x4 (&x)[2], const f32x2* angles) const {
    const bool keys = ROPE && !kind_of(u);
    const unsigned block = (unsigned)slot >> 4, page = block / per_page, within = block - page * per_page;
    const int row = slot & 15;
    uint8_t* scale = scale_of(u, page, within);
    int byte = 0;
    if (row) byte = *scale;
    if (keys) turn_row(x, angles);
    int most = row_max(largest(x, 0));
    const bool odd = most >= 0x7f80;
    if (wave_any(odd)) most = row_max(largest_finite(x, 0));
    const int old = row ? held_exponent(byte) : kScaleMin, e = max(old, block_exponent((uint32_t)most));
    if (lr == 0) *scale = (uint8_t)(e + 127);
    i32x4 y;
    if (wave_any(odd || e == kScaleMax))
      y = over_scale_limited(x, e);
    else
      y = over_scale(x, e);
    char* out = block_of(u, page, within);
    store_row(out + row * p.c.token_stride, keys, y);
    if (row && e > old)
      for (int r = 0; r < kPageRows; ++r)
        if (r != row) rescale(out + r * p.c.token_stride + 16 * lr, e - old);
  }
};

template <int D>
__global__ __launch_bounds__(256) void mala_paged_block_write_kernel(PagedWriteParams p) {
  typename BlockWriter<D, false, false>::Turns none;
  const Turn turn = {};
  BlockWriter<D, false, false>(p, turn).run(blockIdx.x, none);
}

// Keys and values into a block-scaled cache by the first workgroups, queries by the others: two heads
// at a time, since the first kind's registers leave room for half as many wavefronts (16000 tokens,
// 32 + 8 heads, 73.2 / 69.5 us).  In turns, or the queries first, they take longer (75.5, 75.9).
template <int D, bool INTER>
__device__ __forceinline__ void turn_queries(const PagedRopeWriteParams& p) {
  const unsigned nx = (p.q.T + rope_tokens(D) - 1) / rope_tokens(D), i = blockIdx.x - p.kv_groups;
  turn_rows<D, false, false, INTER, false, 2>(p.q, i % nx * rope_tokens(D), (int)(i / nx) * p.q.per);
}

template <int D, bool INTER>
__global__ __launch_bounds__(256) void mala_paged_block_rope_kernel(PagedRopeWriteParams p) {
  if (blockIdx.x < p.kv_groups) {
    __shared__ typename BlockWriter<D, true, INTER>::Turns turns;
    BlockWriter<D, true, INTER>(p.w, p.q.turn).run(blockIdx.x, turns);
  } else {
    turn_queries<D, INTER>(p);
  }
}

// The same for a cache of bf16, or of e4m3 with a scale per head: every row is its own.  HBM-bound: 16000
// tokens, 32 + 8 heads, bf16 75 us, 5.3 TB/s, e4m3 79, 4.6 (a division per value, 8 bytes to a store);
// 64 tokens 3.3 and 3.9.
template <int D, bool E4M3, bool INTER>
__global__ __launch_bounds__(256) void mala_paged_rope_write_kernel(PagedRopeWriteParams p) {
  constexpr int LPR = D / 16, TOK = rope_tokens(D);
  if (blockIdx.x >= p.kv_groups) {
    turn_queries<D, INTER>(p);
    return;
  }
  const unsigned nx = (p.q.T + TOK - 1) / TOK;
  const PagedWriteParams& w = p.w;
  const Turn& turn = p.q.turn;
  const unsigned t = blockIdx.x % nx * TOK + threadIdx.x / LPR, P = w.c.page_size;
  if (t >= p.q.T) return;
  const int slot = w.slots[t], lr = threadIdx.x % LPR;
  if (slot < 0 || (unsigned)slot >= w.c.num_pages * P) return;
  const unsigned page = slot / P, row = slot - page * P;
  const int kind = blockIdx.x / nx % 2, h0 = blockIdx.x / nx / 2 * w.units;
  const Pieces<D, 8, INTER> pc(lr, turn.R);
  float c[8], s[8];
  if (!kind) pc.angles(turn, turn.pos ? turn.pos[t] : (int)t, c, s);
  for (int h = h0; h < min(h0 + w.units, w.c.Hkv); ++h) {
    const char* x = (kind ? w.v : w.k) + t * w.token_stride + h * w.head_stride;
    char* out = (kind ? w.c.v : w.c.k) + page * w.c.page_stride + h * w.c.head_stride + row * w.c.token_stride;
    float v[2][8];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      RawPiece<false, 8> in;
      in.load<false>(x + pc.at[n] * 16);
      in.get(v[n]);
    }
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

static unsigned block_write_groups(PagedWriteParams& p, bool rope) {
  const BlockWritePlan x = block_write_plan(p.T, p.c.Hkv, rope);
  p.chunk = x.chunk;
  p.units = x.units;
  return (unsigned)x.groups;
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
    p.w.units = rope_heads_per_group(p.w.T, p.w.c.Hkv, D);
    p.kv_groups = nx * 2 * ((p.w.c.Hkv + p.w.units - 1) / p.w.units);
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
