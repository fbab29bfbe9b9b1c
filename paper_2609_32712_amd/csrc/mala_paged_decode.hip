// MALA decode of one query token over a paged KV cache (gfx950): the rule of mala_decode.hip
// (splits of the cache, each tested from an empty state, L = n) on 16-row groups of pages.
//
// A wavefront takes a run of tiles (32 keys) of one (sequence, KV head, chunk of up to 16
// query heads of its group), from its last tile down: S^T = K Q^T and O^T += V^T P^T by
// 16x16x32 MFMAs, K and V through the wavefront's own LDS slot.  The wavefronts of a workgroup
// take neighbouring runs and join their (m, l, O) in LDS; a sequence longer than a workgroup's
// share leaves partials that a second launch joins.
//
// What bounds it (MI355X): large calls HBM, 6.2-6.9 TB/s of K and V on 1 GB and more (16 caches
// of 131072 tokens, 8.6 GB: 1.24 ms); calls of 100-300 MB the same and about 10 us of launch, first
// loads (lengths, then table, then K, ~2.5 us), the last workgroups and the join (2.5-4.7 us); small
// ones those alone (one cache of 200 tokens 6.1 us, of 4096 tokens 7.9 + 3.6 us).
//
// A page's 16-row groups are contiguous up to the token stride, so a tile is two buffer
// resources of 16 rows.  Rows at or past the length, and groups of a page whose table entry
// is outside the pool, have a resource of 0 bytes: they read as zeros, move no data, and
// their scores are masked.
//
// Blocks of 16 rows with a scale 2^e (kCacheBlock) are these 16-row groups; the conversion to bf16
// applies the scale, exactly.  They take as long as e4m3 with a scale per head (16 caches of 100000
// tokens 498 us, 6.6 TB/s; 48 ragged ones of up to 8192 75).
#include "mala_device.h"
#include "mala_kernels.h"
#include "mala_paged.h"

namespace mala {

namespace {

// ------------------------------------------------------------------ who works on what
// Only the device knows the lengths, so it shares out the work: every workgroup counts the tiles
// of all sequences, takes blocks of about as many for every workgroup of the target, in units
// of whole splits where tau > 0, and finds its own block (0.6 us for up to 64 sequences).  The
// grid is the bound of what that can come to: a sequence of T_b tiles has max(1, ceil(T_b /
// per_block)) blocks, and with per_block >= total / target they are at most target + B.
struct Share {
  int b, blk;        // sequence, block of it
  int blocks;        // blocks of the sequence
  int first;         // number of its first block among all sequences' (where partials lie)
  int tpw;           // tiles per wavefront (kTeam: per block) in this sequence
  int n;             // its length
};

// The share of block number `at` among all sequences' blocks; b = -1 past the last one.
template <int MODE>
__device__ __forceinline__ Share share_of(const PagedDecParams& p, int at) {
  constexpr int W = MODE == kTeam ? 1 : kPagedWaves;   // runs per block
  const int lane = threadIdx.x & 63;
  const auto tiles = [&](int b) {
    return b < p.B ? (min(max(p.lens[b], 0), p.max_len) + kDecBk - 1) / kDecBk : 0;
  };
  const unsigned unit = MODE == kDense ? 1 : p.unit;
  const int t0 = tiles(lane);          // of the first 64 sequences
  unsigned total = 0;
  int longest = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int t = b0 ? tiles(b0 + lane) : t0;
    total += __builtin_amdgcn_readlane(wave_scan(t), 63);
    longest = max(longest, wave_max(t));
  }
  const unsigned per_block =
      paged_block_tiles(total, longest, p.B, p.target, p.ragged, p.min_tpw, unit, W);
  Share s = {-1, 0, 1, 0, 0, 0};
  int before = 0;                      // blocks of the sequences before
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int t = b0 ? tiles(b0 + lane) : t0, here = min(64, p.B - b0);
    const int nb = lane < here ? paged_blocks_of(t, per_block) : 0;
    const int end = wave_scan(nb), all = __builtin_amdgcn_readlane(end, 63);
    if (at < before + all) {
      // even runs within a sequence.  Its blocks but the last, which are full, take the places [from, from +
      // nb - 1) of these 64 sequences' blocks, its last one, of what is left of it, the place `last`:
      // the blocks of the most tiles first
      const int tpw = paged_run_tiles(t, max(nb, 1), unit, W), full = W * tpw;
      int from = end - nb, last = end - 1;
      if (p.sorted && __builtin_amdgcn_ballot_w64(lane < here && tpw > 4)) {
        const int cls = paged_run_class(full, per_block, 1);
        const int cls_last = paged_run_class(t - (nb - 1) * full, per_block, 1);
        int base = 0;
#pragma unroll
        for (int c = kPagedClasses - 1; c >= 0; --c) {
          const int n = nb == 0 ? 0 : (cls == c ? nb - 1 : 0) + (cls_last == c ? 1 : 0);
          const int e = wave_scan(n), at_c = base + e - n;
          if (cls == c) from = at_c;
          if (cls_last == c) last = base + e - 1;
          base += __builtin_amdgcn_readlane(e, 63);
        }
      }
      const int place = at - before;
      const bool mine = lane < here && ((from <= place && place < from + nb - 1) || place == last);
      const int i = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine));
      s.b = b0 + i;
      s.blocks = __builtin_amdgcn_readlane(nb, i);
      s.first = before + __builtin_amdgcn_readlane(end, i) - s.blocks;
      s.blk = place == __builtin_amdgcn_readlane(last, i) ? s.blocks - 1
                                                           : place - __builtin_amdgcn_readlane(from, i);
      s.tpw = __builtin_amdgcn_readlane(tpw, i);
      s.n = min(max(p.lens[s.b], 0), p.max_len);
      return s;
    }
    before += all;
  }
  return s;
}

// The next bf16 term of eight probabilities; x becomes what is left.  Three terms hold all 24 bits
// of an fp32, whatever the type of the output, so that a bf16 output is the fp32 one rounded once.
// (Two terms, 16 bits, save time only where several chunks of heads share K and V: us per call with
// two / three 49.9 / 50.0 for 16 ragged 8192-token caches, 41.1 / 41.2 for 64 ragged e4m3 ones, 1278 /
// 1278 for 16 of 131072 tokens, 33.8 / 36.4 for 16 of 8192 with 64 heads on 2.)
__device__ __forceinline__ bf16x8 take_bf16x8(float (&x)[8]) {
#pragma clang fp contract(off)
  i32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t h = __builtin_bit_cast(
        uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
    x[2 * i] -= __uint_as_float(h << 16);          // exact: a bf16 is the upper half of an fp32
    x[2 * i + 1] -= __uint_as_float(h & 0xffff0000u);
    u[i] = (int)h;
  }
  return __builtin_bit_cast(bf16x8, u);
}

// Reductions over the four 16-lane rows of a wavefront (lanes of equal lane % 16).
__device__ __forceinline__ float rows_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float rows_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// a b as an fp32, whatever takes it
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// The rule's state of one split and head: m, l, reference and normaliser of the keys retained.
// kChain and kTeam decide by these functions alone.  Which of the two a call takes goes by its
// batch, and what is retained must not: so each operation rounds as it is written here (fused ones
// are written out, here and wherever a product meets a sum below, and the compiler adds none).
struct SplitState {
  float m = kNegInf, l = 0.f;
  __device__ __forceinline__ float run() const { return m + fast_log2(l); }
  // of a tile with the largest score mt (l = 0: the split's first one)
  __device__ __forceinline__ bool retains(float mt, float run, float thr2) const {
    return l == 0.f || paged_retains(mt, run, thr2);
  }
  __device__ __forceinline__ bool may_retain(float mt, float run, float thr2) const {
    return l == 0.f || paged_may_retain(mt, run, thr2);
  }
  // adds a tile: `sum` of its 2^(score - mt), or of scores of -inf alone 0
  __device__ __forceinline__ void add(float mt, float sum) {
#pragma clang fp contract(off)
    const float own = mt == kNegInf ? 0.f : mt, top = fmaxf(m, mt), ref = top == kNegInf ? 0.f : top;
    l = __builtin_fmaf(l, fast_exp2(m - ref), sum * fast_exp2(own - ref));
    m = top;
  }
};

// Where a tile's pieces of 8 values lie in LDS: rows D + 16 apart, and within a row (SWAP: of 128 bytes
// in the cache, where a lane has two neighbouring pieces to store) the even pieces in front of the odd
// ones, these in pairs swapped.  K reads (a phase takes rows 0-3 and 12-15 of one piece with 4-11 of
// the next), transposed V reads and stores (128 bytes at a time) then find no two lanes on one bank.
// With rows D + 8 apart and the pieces in order LDS was busy 384 instead of 192 cycles per tile of
// bytes; us per call before / now: 48 ragged caches of up to 8192 tokens 71.5 / 70.0, 16 of 8192 with 64
// heads on 2 27.5 / 26.9.
template <int D, bool SWAP>
struct Layout {
  static constexpr int LD = D == 128 ? D + 16 : D + 8;    // (D = 64: a wavefront per SIMD less, 52 / 60 us)
  // element of piece n of a row
  static __device__ __forceinline__ constexpr int at(int n) {
    return 8 * (!SWAP ? n : n % 2 ? D / 16 + (n / 2 ^ 1) : n / 2);
  }
  // piece 4 kk + g: k_lane(g) + k_step(kk)
  static __device__ __forceinline__ int k_lane(int g) { return at(g); }
  static constexpr int k_step(int kk) { return SWAP ? 16 * kk : 32 * kk; }
  // values 16 db + 4 j .. + 3: v_lane(j, db odd?) + v_step(db)
  static __device__ __forceinline__ int v_lane(int j, int odd) {
    return SWAP ? (j >> 1 ? D / 2 + (odd ? -8 : 8) : 0) + 4 * (j & 1) : 4 * j;
  }
  static constexpr int v_step(int db) { return SWAP ? 8 * db : 16 * db; }
};

template <int D, int FMT, int MODE>
__global__ __launch_bounds__(kPagedWaves * 64, 2) void mala_paged_decode_kernel(PagedDecParams p) {
  constexpr int W = kPagedWaves;
  constexpr bool DENSE = MODE == kDense, TEAM = MODE == kTeam;
  constexpr bool E4M3 = FMT == kCacheE4M3, BLOCK = FMT == kCacheBlock, BYTES = E4M3 || BLOCK;
  constexpr int KS = D / 32;             // k-steps of 32 over head_dim
  constexpr int NDB = D / 16;            // 16-row blocks of O^T
  using Lay = Layout<D, FMT != kCacheBf16 && D == 128>;
  constexpr int LD = Lay::LD;
  constexpr int CPR = D / (BYTES ? 16 : 8);   // 16-byte chunks per row of the cache
  constexpr int RPI = 64 / CPR;          // rows per load instruction
  constexpr int IPG = kPageRows / RPI;   // load instructions per 16-row group
  static_assert(IPG >= 1, "a load instruction stays within a group");
  // a K or V tile of 32 rows of bf16, later the wavefront's 16 x D accumulator in fp32
  __shared__ __attribute__((aligned(16))) bf16 slot[W][kDecBk * LD];
  __shared__ float refs[W][16], sums[W][16];
  __shared__ int counts[W][16];
  __shared__ f32x2 tests[TEAM ? 2 : 1][W][16];       // kTeam: a round's maxima and sums

  const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = p.c.Hkv, grp = p.Hq / Hkv;
  // Workgroups are dealt to the CUs in turn, a round of 256 at a time, and the share of HBM that
  // a CU gets is its own: longest first, and every other round backwards, gives the CUs about
  // as many tiles each.
  const int round = blockIdx.x / kNumCus, spot = blockIdx.x % kNumCus;
  const int place = round * kNumCus + (round % 2 ? kNumCus - 1 - spot : spot);
  // (block of a sequence, KV head), and chunk of the KV head's query heads
  const int item = paged_item(place, p.nchunk), chunk = paged_chunk(place, p.nchunk);
  Share sh;
  if (p.sorted) {
    __shared__ Share plan;
    if (w == 0) {
      const Share x = share_of<MODE>(p, item / Hkv);
      if (lane == 0) plan = x;
    }
    __syncthreads();
    sh.b = __builtin_amdgcn_readfirstlane(plan.b);
    sh.blk = __builtin_amdgcn_readfirstlane(plan.blk);
    sh.blocks = __builtin_amdgcn_readfirstlane(plan.blocks);
    sh.first = __builtin_amdgcn_readfirstlane(plan.first);
    sh.tpw = __builtin_amdgcn_readfirstlane(plan.tpw);
    sh.n = __builtin_amdgcn_readfirstlane(plan.n);
  } else {
    sh = share_of<MODE>(p, item / Hkv);
  }
  if (sh.b < 0) return;                              // the same for the whole workgroup
  const int hkv = item % Hkv, b = sh.b;
  const int nh = min(16, grp - 16 * chunk), h0 = hkv * grp + 16 * chunk;
  const int n = sh.n, T = (n + kDecBk - 1) / kDecBk;
  const int t_lo = min(T, (TEAM ? sh.blk : sh.blk * W + w) * sh.tpw), t_hi = min(T, t_lo + sh.tpw);
  const bool head_valid = col < nh;
  const uint32_t ts = (uint32_t)p.c.token_stride;

  // Where the 64 16-row groups below group `g_top` are (32 tiles): lane i holds, of group g_top - i,
  // the byte offset from the pool's start and how many of its rows are there (0: past the
  // length, or of a page whose entry is outside the pool).
  uint32_t off_lo = 0, off_hi = 0;
  int rows = 0;
  uint32_t kscale = 0, vscale = 0;     // kCacheBlock: of the group's K and V, as bits of an fp32
  const int32_t* entry = p.table + (long)b * p.W;
  const unsigned gpp = p.c.page_size / kPageRows;
  const auto find_groups = [&](int g_top) {
    const int gr = g_top - lane;
    rows = gr >= 0 ? max(0, min(kPageRows, n - gr * kPageRows)) : 0;
    const unsigned page = (unsigned)max(gr, 0) / gpp, within = (unsigned)max(gr, 0) - page * gpp;
    const int number = rows > 0 ? entry[page] : -1;
    rows = (unsigned)number < (unsigned)p.c.num_pages ? rows : 0;
    const uint64_t off = rows ? (uint64_t)number * (uint64_t)p.c.page_stride +
                                    (uint64_t)hkv * (uint64_t)p.c.head_stride +
                                    (uint64_t)(within * kPageRows) * ts
                              : 0;
    off_lo = (uint32_t)off;
    off_hi = (uint32_t)(off >> 32);
    if constexpr (BLOCK) {
      kscale = vscale = 0x3f800000;
      if (rows) {
        const int64_t at = ((int64_t)number * Hkv + hkv) * gpp + within;
        kscale = block_scale_bits(p.c.kb[at]);
        vscale = block_scale_bits(p.c.vb[at]);
      }
    }
  };
  find_groups(2 * t_hi - 1);

  // q rows of the heads (zeros for the columns that have none)
  bf16x8 qreg[KS];
  {
    const auto r = make_rsrc(p.q + ((long)b * p.Hq + h0) * D, (uint32_t)(nh * D * 2));
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
      qreg[kk] = __builtin_bit_cast(
          bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, (col * D + 32 * kk + 8 * g) * 2, 0, 0));
  }
  // scores are scale2 x (K row . q), scale2 > 0: a negative scale goes into q, and one of 0 stays
  // large enough to keep a masked score at -inf
  float scale2 = p.scale2;
  if (E4M3 && p.c.ks) {
    scale2 *= p.c.ks[hkv];
    if (scale2 < 0.f) {
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qreg[kk] = -qreg[kk];
      scale2 = -scale2;
    }
    if (scale2 == 0.f) scale2 = 1e-37f;
  }
  // for the join: where the sequence's partials lie
  if (sh.blk == 0 && hkv == 0 && chunk == 0 && threadIdx.x == 0 && p.nblk > p.B)
    p.plan[b] = make_int2(sh.first, sh.blocks);
  const float thr2 = DENSE ? 0.f : p.log2tau - log2f((float)n);    // L = n

  // a tile's two groups: where they start, and how many of their rows are there
  struct Place {
    uint64_t off0, off1;
    int rows0, rows1;
    int lane;            // that holds the upper group (kCacheBlock)
    uint32_t ks0, ks1, vs0, vs1;
  };
  int in = 0;                            // lane of the next tile's upper group
  // where tile t is, the one below the last asked for (kTeam: any below it); nowhere below t_end
  int top = t_hi - 1;                    // its lane 0 holds this tile (kTeam)
  const auto next_tile = [&](int t, int t_end) {
    Place x = {0, 0, 0, 0, 0, 0, 0, 0, 0};
    if (t < t_end) return x;
    if constexpr (TEAM) {
      if (top - t >= 32) {
        find_groups(2 * t + 1);
        top = t;
      }
      in = 2 * (top - t);
    } else if (in == 64) {
      find_groups(2 * t + 1);
      in = 0;
    }
    x.off1 = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, in) << 32 |
             (uint32_t)__builtin_amdgcn_readlane(off_lo, in);
    x.rows1 = __builtin_amdgcn_readlane(rows, in);
    x.off0 = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, in + 1) << 32 |
             (uint32_t)__builtin_amdgcn_readlane(off_lo, in + 1);
    x.rows0 = __builtin_amdgcn_readlane(rows, in + 1);
    x.lane = in;
    in += 2;
    return x;
  };
  // A place's scales.  They are loaded behind its offsets, and read here once the place's turn has
  // come (before the next lookup), so that its K and V loads do not wait for them.
  const auto take_scales = [&](Place& x) {
    if constexpr (BLOCK) {
      x.ks1 = __builtin_amdgcn_readlane(kscale, x.lane);
      x.vs1 = __builtin_amdgcn_readlane(vscale, x.lane);
      x.ks0 = __builtin_amdgcn_readlane(kscale, x.lane + 1);
      x.vs0 = __builtin_amdgcn_readlane(vscale, x.lane + 1);
    }
  };

  uint32_t lane_off[IPG];
#pragma unroll
  for (int i = 0; i < IPG; ++i) {
    lane_off[i] = (lane / CPR + i * RPI) * ts + (lane % CPR) * 16;
    asm("" : "+v"(lane_off[i]));         // kept, not computed again at every load
  }
  typedef bf16x8 Tile[2 * IPG];          // raw bytes (16 per lane and instruction)
  const auto load_tile = [&](const char* base, const Place& at, bool want, Tile& x) {
    const auto r0 = make_rsrc(base + at.off0, want ? at.rows0 * ts : 0u);
    const auto r1 = make_rsrc(base + at.off1, want ? at.rows1 * ts : 0u);
#pragma unroll
    for (int i = 0; i < IPG; ++i) {
      x[i] = buf_load8_stream(r0, lane_off[i]);
      x[IPG + i] = buf_load8_stream(r1, lane_off[i]);
    }
  };
  // A tile's rows to LDS.  One wavefront's LDS accesses complete in issue order, so K and V
  // tiles can follow each other in one slot without waits.
  bf16* mine = slot[w];
  const auto to_lds = [&](const Tile& x, uint32_t scale0, uint32_t scale1) {
#pragma unroll
    for (int i = 0; i < 2 * IPG; ++i) {
      const int r = i * RPI + lane / CPR, c = lane % CPR;
      if constexpr (BYTES) {
        const i32x4 raw = __builtin_bit_cast(i32x4, x[i]);
        const float f = BLOCK ? __uint_as_float(i < IPG ? scale0 : scale1) : 1.f;
        i32x4 y[2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          y[k / 2][2 * (k % 2)] = __builtin_bit_cast(
              int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[k], f, false));
          y[k / 2][2 * (k % 2) + 1] = __builtin_bit_cast(
              int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[k], f, true));
        }
        store8(mine + r * LD + Lay::at(2 * c), __builtin_bit_cast(bf16x8, y[0]));
        store8(mine + r * LD + Lay::at(2 * c + 1), __builtin_bit_cast(bf16x8, y[1]));
      } else {
        store8(mine + r * LD + c * 8, x[i]);
      }
    }
  };

  const int k_lane = Lay::k_lane(g), v_even = Lay::v_lane(col & 3, 0), v_odd = Lay::v_lane(col & 3, 1);

  // Products of the K tile in LDS with this lane's head (before scale2): s[0..3] keys 4 g + r,
  // s[4..7] keys 16 + 4 g + r; keys that are not there -inf.  Returns the scaled maximum.
  const auto scores = [&](const Place& at, float (&s)[8]) {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      s0 = mfma16(load8(mine + col * LD + k_lane + Lay::k_step(kk)), qreg[kk], s0);
      s1 = mfma16(load8(mine + (16 + col) * LD + k_lane + Lay::k_step(kk)), qreg[kk], s1);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[r] = s0[r];
      s[4 + r] = s1[r];
    }
    if (at.rows0 + at.rows1 < kDecBk) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (4 * g + r >= at.rows0) s[r] = kNegInf;
        if (4 * g + r >= at.rows1) s[4 + r] = kNegInf;
      }
    }
    float x = fmaxf(s[0], s[4]);
#pragma unroll
    for (int r = 1; r < 4; ++r) x = fmaxf(x, fmaxf(s[r], s[4 + r]));
    return rounded_product(rows_max(x), scale2);
  };

  // m, l: reference and normaliser of what this wavefront retained (l of this lane's keys;
  // the rows are added at the end).
  float m = kNegInf, l = 0.f;
  f32x4 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  // moves the reference up to m_new (most tiles leave every head's where it is)
  const auto raise = [&](float m_new) {
    if (!wave_any(m_new > m)) return;
    const float alpha = m_new > m ? fast_exp2(m - m_new) : 1.f;
    l *= alpha;
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[db] *= alpha;
    m = m_new;
  };
  // adds the V tile in LDS, weighted
  const auto add_values = [&](float (&x)[8]) {
    const bf16x8 ph = take_bf16x8(x), pl = take_bf16x8(x), pr = take_bf16x8(x);
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      const bf16* vrow = mine + (4 * g + (col >> 2)) * LD + (db % 2 ? v_odd : v_even) + Lay::v_step(db);
      const bf16x8 a = cat(lds_read_tr(vrow), lds_read_tr(vrow + 16 * LD));
      acc[db] = mfma16(a, ph, acc[db]);
      acc[db] = mfma16(a, pl, acc[db]);
      acc[db] = mfma16(a, pr, acc[db]);
    }
  };
  int cnt = 0;
  unsigned legal = 0, vfetch = 0, vloads = 0;
  unsigned long long hsum = 0;
  int split_lo = TEAM ? max(t_hi - 1, 0) / p.unit * p.unit : 0;   // first tile of the split
  Tile kr, vr;
  Place at = next_tile(TEAM ? t_hi - 1 - w : t_hi - 1, TEAM ? split_lo : t_lo);
  load_tile(p.c.k, at, true, kr);
  load_tile(p.c.v, at, true, vr);
  take_scales(at);

  if constexpr (DENSE) {
    // every tile counts: K and V of the next one load while a tile is worked on.  (Columns
    // without a head have zero queries; what they hold is never stored.)
    for (int t = t_hi - 1; t >= t_lo; --t) {
      const Place next = next_tile(t - 1, t_lo);
      to_lds(kr, at.ks0, at.ks1);
      load_tile(p.c.k, next, true, kr);
      float s[8];
      const float mt = scores(at, s);
      raise(fmaxf(m, mt));
      const float shift = m == kNegInf ? 0.f : m;       // scores of -inf alone add 0
      to_lds(vr, at.vs0, at.vs1);
      load_tile(p.c.v, next, true, vr);
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = fast_exp2(__builtin_fmaf(s[r], scale2, -shift));
      l += ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
      add_values(s);
      const bool here = at.rows0 + at.rows1 > 0;
      legal += here ? 1u : 0u;
      if (p.counters && here) hsum += tile_hash(b, h0 + col, 0, t);
      at = next;
      take_scales(at);
    }
    cnt = legal;
    vfetch = vloads = legal;
  } else if constexpr (TEAM) {
    // What bounds a call of few splits is the chain of a split's tiles.  Here the wavefronts score
    // W tiles at once and publish each tile's maximum and sum per head (against that maximum);
    // behind a barrier every wavefront takes the W tests in order, carrying the split's state,
    // and adds its tile's values if its own was retained.  K and V of the next round load
    // meanwhile; V is fetched for every tile.
    SplitState state;
    for (int t0 = t_hi - 1, round = 0; t0 >= t_lo; ++round) {
      int t_next = t0 - W, lo_next = split_lo;
      if (t_next < split_lo) {               // the split below
        t_next = split_lo - 1;
        lo_next = split_lo - p.unit;
      }
      const Place next = next_tile(t_next - w, max(lo_next, t_lo));
      to_lds(kr, at.ks0, at.ks1);
      load_tile(p.c.k, next, true, kr);
      float s[8];
      const float mt = scores(at, s), own = mt == kNegInf ? 0.f : mt;
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = fast_exp2(__builtin_fmaf(s[r], scale2, -own));
      const float ps = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
      const float all = rows_sum(ps);
      const bool here = at.rows0 + at.rows1 > 0;
      if (g == 0) tests[round & 1][w][col] = f32x2{mt, here ? all : -1.f};
      to_lds(vr, at.vs0, at.vs1);
      load_tile(p.c.v, next, true, vr);
      __syncthreads();
      bool mine = false;
#pragma unroll
      for (int u = 0; u < W; ++u) {
        const f32x2 x = tests[round & 1][u][col];     // (a sum below 0: no key of the tile is there)
        const bool demand = head_valid && !(x[1] < 0.f) && state.retains(x[0], state.run(), thr2);
        if (u == w) mine = demand;
        if (demand) state.add(x[0], x[1]);
      }
      legal += here ? 1u : 0u;
      if (wave_any(mine)) {
        ++vloads;
        raise(mine ? fmaxf(m, mt) : m);
        const float shift = m == kNegInf ? 0.f : m, f = mine ? fast_exp2(own - shift) : 0.f;
        if (mine) {
          l = __builtin_fmaf(ps, f, l);
          ++cnt;
          if (p.counters) hsum += tile_hash(b, h0 + col, 0, t0 - w);
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) s[r] = mine ? s[r] * f : 0.f;
        add_values(s);
      }
      if (lo_next != split_lo) state = SplitState();
      t0 = t_next;
      split_lo = lo_next;
      at = next;
      take_scales(at);
    }
    vfetch = legal;
  } else if (t_hi > t_lo) {
    // While tile t is worked on, K of t - 1 is in registers or on its way (its scores are taken
    // first), K of t - 2 and V of t load.  V of t - 1 is fetched when the state before tile t's
    // update may retain it.
    SplitState state;                        // of the split being tested
    float s[8], sn[8];
    int left = (t_hi - 1) % p.unit + 1;      // tiles of the split from t down
    Place next = next_tile(t_hi - 2, t_lo);
    to_lds(kr, at.ks0, at.ks1);
    load_tile(p.c.k, next, true, kr);
    float mt = scores(at, s);
    take_scales(next);
    vfetch = at.rows0 + at.rows1 > 0;
    for (int t = t_hi - 1; t >= t_lo; --t) {
      const Place after = next_tile(t - 2, t_lo);
      to_lds(kr, next.ks0, next.ks1);        // K of t - 1 (zeros past the run's first tile)
      load_tile(p.c.k, after, true, kr);
      const float mtn = scores(next, sn);
      const bool here = at.rows0 + at.rows1 > 0, there = next.rows0 + next.rows1 > 0;
      const float run = state.run();
      const bool demand = head_valid && here && state.retains(mt, run, thr2);
      const bool last = --left == 0;         // the next tile starts a split: always retained
      const bool hint =
          there && (last || wave_any(head_valid && state.may_retain(mtn, run, thr2)));
      const bool any = wave_any(demand);
      if (any) to_lds(vr, at.vs0, at.vs1);
      load_tile(p.c.v, next, hint, vr);
      legal += here ? 1u : 0u;
      vfetch += hint ? 1u : 0u;
      if (any) {
        ++vloads;
        raise(demand ? fmaxf(m, mt) : m);
        // weights against the tile's own maximum, for the split's state, and from there to the
        // run's reference
        const float shift = m == kNegInf ? 0.f : m;     // a tile of -inf scores adds 0
        const float own = mt == kNegInf ? 0.f : mt, f = demand ? fast_exp2(own - shift) : 0.f;
#pragma unroll
        for (int r = 0; r < 8; ++r)
          s[r] = demand ? fast_exp2(__builtin_fmaf(s[r], scale2, -own)) : 0.f;
        const float ps = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
        const float all = rows_sum(ps);
        if (demand) {
          state.add(mt, all);
          ++cnt;
          if (p.counters) hsum += tile_hash(b, h0 + col, 0, t);
        }
        l = __builtin_fmaf(ps, f, l);
#pragma unroll
        for (int r = 0; r < 8; ++r) s[r] *= f;
        add_values(s);
      }
      if (last) {
        state = SplitState();
        left = p.unit;
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = sn[r];
      mt = mtn;
      at = next;
      next = after;
      take_scales(next);
    }
  }
  l = rows_sum(l);

  // join the wavefronts: per head a common reference and normaliser, then every accumulator's
  // share of the output, added up
  if (g == 0) {
    refs[w][col] = m;
    sums[w][col] = l;
    counts[w][col] = cnt;
  }
  __syncthreads();
  float M = kNegInf, L = 0.f;
#pragma unroll
  for (int u = 0; u < W; ++u) M = fmaxf(M, refs[u][col]);
  const float top_m = M;
  if (M == kNegInf) M = 0.f;
#pragma unroll
  for (int u = 0; u < W; ++u) L = __builtin_fmaf(sums[u][col], fast_exp2(refs[u][col] - M), L);
  const long part = (long)(sh.first + sh.blk) * p.Hq + h0;   // of the block's first head
  {
    // (0 for a wavefront without keys)
    const float f = L != 0.f ? fast_exp2(m - M) * (E4M3 && p.c.vs ? p.c.vs[hkv] : 1.f) / L : 0.f;
    float* out = reinterpret_cast<float*>(mine);
    static_assert(sizeof(slot[0]) >= 16 * D * sizeof(float), "an accumulator fits a tile");
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      *reinterpret_cast<f32x4*>(out + (db * 64 + lane) * 4) = acc[db] * f;
  }
  if (threadIdx.x < nh) {
    int kept = 0;
#pragma unroll
    for (int u = 0; u < W; ++u) kept += counts[u][col];
    if (sh.blocks == 1) {
      const long bh = (long)b * p.Hq + h0 + col;
      p.lse[bh] = L != 0.f ? (M + fast_log2(L)) * kLn2 : kNegInf;
      if (p.head_tiles) p.head_tiles[bh] = kept;
    } else {
      *reinterpret_cast<f32x4*>(p.part + (part + col) * (D + kDecStride) + D) =
          f32x4{top_m, L, __int_as_float(kept), 0.f};
    }
  }
  __syncthreads();
  static_assert(NDB * 64 % (W * 64) == 0, "whole rounds of the workgroup's threads");
#pragma unroll
  for (int i0 = 0; i0 < NDB * 64; i0 += W * 64) {
    const int i = i0 + threadIdx.x, c = i & 15, d = 16 * (i >> 6) + 4 * ((i & 63) >> 4);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < W; ++u)
      o += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(slot[u]) + i * 4);
    if (c >= nh) continue;
    if (sh.blocks == 1)
      store_out4(p.o, ((long)b * p.Hq + h0 + c) * D + d, o, p.o_bf16);
    else
      *reinterpret_cast<f32x4*>(p.part + (part + c) * (D + kDecStride) + d) = o;
  }
  if (p.counters) {
    if (head_valid && g == 0 && cnt) {
      atomicAdd(&p.counters[kCntRetained], (unsigned long long)cnt);
      atomicAdd(&p.counters[kCntSlots], (unsigned long long)cnt * kDecBk);
      atomicAdd(&p.counters[kCntSetHash], hsum);
    }
    if (lane == 0 && legal) {
      atomicAdd(&p.counters[kCntLegal], (unsigned long long)legal * nh);
      atomicAdd(&p.counters[kCntVTiles], (unsigned long long)vfetch);
      atomicAdd(&p.counters[kCntVNeeded], (unsigned long long)vloads);
    }
  }
}

__device__ __forceinline__ f32x4 fma4(f32x4 a, float f, f32x4 c) {
  return __builtin_elementwise_fma(a, f32x4{f, f, f, f}, c);
}

// Joins the partials (O_s / l_s, m_s, l_s, count) of the sequences that have more than one block:
// l = sum_s 2^(m_s - m) l_s, o = sum_s 2^(m_s - m) l_s (O_s / l_s) / l, a workgroup per query head.
// LPR lanes read a partial row 16 bytes each, the workgroup's NG groups of LPR lanes take the
// parts in turn.  Latency-bound: 2.5-4.7 us (where the sequence's parts lie, then their states and
// rows at once).
constexpr int kJoinThreads = 256;
template <int D>
__global__ __launch_bounds__(kJoinThreads) void mala_paged_join_kernel(PagedDecParams p) {
  constexpr int LPR = D / 4, NG = kJoinThreads / LPR, REC = D + kDecStride;
  __shared__ __attribute__((aligned(16))) f32x4 rows[kJoinThreads];
  __shared__ f32x2 state[NG];
  __shared__ int counts[NG];
  const int tid = threadIdx.x, grp = tid / LPR, cl = tid % LPR;
  const int b = blockIdx.x / p.Hq, h = blockIdx.x % p.Hq;
  const int2 plan = p.plan[b];
  const int nb = plan.y;
  if (nb <= 1) return;                   // the decode kernel wrote the outputs
  const long step = (long)p.Hq * REC;
  const float* pp = p.part + (long)plan.x * step + (long)h * REC;
  float m = kNegInf, z = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  int kept = 0;
  // four of the group's parts at a time: every lane takes their states (one address for the
  // group's lanes) and its piece of their rows
  for (int s0 = grp; s0 < nb; s0 += 4 * NG) {
    f32x4 x[4], r[4];
    float m_new = m;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + u * NG;
      const float* part = pp + (long)(s < nb ? s : s0) * step;
      x[u] = *reinterpret_cast<const f32x4*>(part + D);
      r[u] = *reinterpret_cast<const f32x4*>(part + 4 * cl);
      if (s >= nb) x[u] = f32x4{kNegInf, 0.f, 0.f, 0.f};
      m_new = fmaxf(m_new, x[u][0]);
    }
    const float ref = m_new == kNegInf ? 0.f : m_new, alpha = fast_exp2(m - ref);
    m = m_new;
    acc *= alpha;
    z *= alpha;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      // f: 0 for a part without keys, and past the last part, where r is the row of part s0 again
      const float e = fast_exp2(x[u][0] - ref), f = x[u][1] * e;
      z = __builtin_fmaf(x[u][1], e, z);
      kept += __float_as_int(x[u][2]);
      acc = fma4(r[u], f, acc);
    }
  }
  rows[tid] = acc;                       // the groups' sums
  if (cl == 0) {
    state[grp] = f32x2{m, z};
    counts[grp] = kept;
  }
  __syncthreads();
  if (grp) return;
  m = kNegInf;
#pragma unroll
  for (int u = 0; u < NG; ++u) m = fmaxf(m, state[u][0]);
  const float ref = m == kNegInf ? 0.f : m;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
  z = 0.f;
  kept = 0;
#pragma unroll
  for (int u = 0; u < NG; ++u) {
    const float f = fast_exp2(state[u][0] - ref);
    z = __builtin_fmaf(state[u][1], f, z);
    acc = fma4(rows[u * LPR + cl], f, acc);
    kept += counts[u];
  }
  const long bh = blockIdx.x;
  store_out4(p.o, bh * D + 4 * cl, acc * (z != 0.f ? 1.f / z : 0.f), p.o_bf16);
  if (cl == 0) {
    p.lse[bh] = z != 0.f ? (ref + fast_log2(z)) * kLn2 : kNegInf;
    if (p.head_tiles) p.head_tiles[bh] = kept;
  }
}

// ------------------------------------------------------------------ launches
template <int D, int FMT, int MODE>
void launch_t(const PagedDecParams& p, hipStream_t st) {
  const dim3 grid(paged_grid(p.nblk * p.c.Hkv, p.nchunk)), wg(kPagedWaves * 64);
  hipLaunchKernelGGL((mala_paged_decode_kernel<D, FMT, MODE>), grid, wg, 0, st, p);
  if (p.nblk > p.B)
    hipLaunchKernelGGL(mala_paged_join_kernel<D>, dim3((unsigned)(p.B * p.Hq)), dim3(kJoinThreads), 0,
                       st, p);
}
template <int D, int FMT>
void launch_e(const PagedDecParams& p, int mode, hipStream_t st) {
  if (mode == kDense)
    launch_t<D, FMT, kDense>(p, st);
  else if (mode == kTeam)
    launch_t<D, FMT, kTeam>(p, st);
  else
    launch_t<D, FMT, kChain>(p, st);
}

template <int D>
void launch_d(const PagedDecParams& p, int mode, hipStream_t st) {
  if (p.c.fmt == kCacheBlock)
    launch_e<D, kCacheBlock>(p, mode, st);
  else if (p.c.fmt == kCacheE4M3)
    launch_e<D, kCacheE4M3>(p, mode, st);
  else
    launch_e<D, kCacheBf16>(p, mode, st);
}

}  // namespace

hipError_t launch_paged_decode(PagedDecParams p, int D, int split_tokens, hipStream_t st) {
  const PagedPlan x = paged_plan(p.B, p.Hq, p.c.Hkv, D, p.c.fmt != kCacheBf16, p.max_len, split_tokens,
                                 p.log2tau == kNegInf);
  p.target = x.target;
  p.ragged = x.ragged;
  p.unit = x.unit;
  p.min_tpw = x.min_tpw;
  p.nblk = x.blocks;
  p.nchunk = x.nchunk;
  p.sorted = p.B > 1 && (long)p.nblk * p.c.Hkv * p.nchunk > kNumCus;
  D == 128 ? launch_d<128>(p, x.mode, st) : launch_d<64>(p, x.mode, st);
  return hipGetLastError();
}

}  // namespace mala
