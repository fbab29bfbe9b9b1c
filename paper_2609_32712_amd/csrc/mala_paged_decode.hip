// MALA decode of one query token over a paged KV cache (gfx950): the rule of mala_decode.hip
// (splits of the cache, each tested from an empty state, L = n) on 16-row groups of pages.
//
// A workgroup of kPagedWaves wavefronts takes consecutive splits of one (sequence, KV head,
// chunk of up to 16 query heads of its group), a split per wavefront: tiles of 32 keys from
// the split's last one down, S^T = K Q^T and O^T += V^T P^T by 16x16x32 MFMAs, K and V through
// the wavefront's own LDS slot.  The wavefronts' (m, l, O) are joined in LDS; sequences longer
// than a workgroup's share leave partials that a second launch joins.
//
// A page's 16-row groups are contiguous up to the token stride, so a tile is two buffer
// resources of 16 rows.  Rows at or past the length, and groups of a page whose table entry
// is outside the pool, have a resource of 0 bytes: they read as zeros, move no data, and
// their scores are masked.
#include "mala_device.h"
#include "mala_kernels.h"
#include "mala_paged.h"

namespace mala {

namespace {

constexpr int kPagedWaves = 4;

// x ~= hi + lo + rest to 24 bits: fp32 outputs keep fp32's accuracy (with two terms the
// probabilities carry 16 bits, ~3e-6 relative, fine below a bf16 output's 2^-9)
__device__ __forceinline__ bf16x8 rest_bf16x8(const float* x, bf16x8 hi, bf16x8 lo) {
#pragma clang fp contract(off)
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (bf16)((x[i] - (float)hi[i]) - (float)lo[i]);
  return r;
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kPagedWaves * 64) void mala_paged_decode_kernel(PagedDecParams p) {
  constexpr int KS = D / 32;             // k-steps of 32 over head_dim
  constexpr int NDB = D / 16;            // 16-row blocks of O^T
  constexpr int LD = D + 8;
  constexpr int CPR = D / (E4M3 ? 16 : 8);   // 16-byte chunks per row of the cache
  constexpr int RPI = 64 / CPR;          // rows per load instruction
  constexpr int IPG = kPageRows / RPI;   // load instructions per 16-row group
  static_assert(IPG >= 1, "a load instruction stays within a group");
  // a K or V tile of 32 rows of bf16, later the wavefront's 16 x D accumulator in fp32
  __shared__ __attribute__((aligned(16))) bf16 slot[kPagedWaves][kDecBk * LD];
  __shared__ float refs[kPagedWaves][16], sums[kPagedWaves][16];
  __shared__ int counts[kPagedWaves][16];

  const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = p.c.Hkv, grp = p.Hq / Hkv, items = p.B * Hkv * p.nchunk;
  const int blk = blockIdx.x / items, item = blockIdx.x % items;
  const int chunk = item % p.nchunk, bhk = item / p.nchunk;
  const int b = bhk / Hkv, hkv = bhk % Hkv;
  const int nh = min(16, grp - 16 * chunk);
  const int n = min(max(p.lens[b], 0), p.max_len);
  const int T = (n + kDecBk - 1) / kDecBk;
  const int wg_lo = blk * kPagedWaves * p.tps;       // first tile of the workgroup
  if (blk > 0 && wg_lo >= T) return;                 // past the sequence: no partial
  const int t_lo = min(T, wg_lo + w * p.tps), t_hi = min(T, t_lo + p.tps);
  const float thr2 = p.log2tau - log2f((float)n);    // L = n
  const bool head_valid = col < nh;
  const int hq = hkv * grp + 16 * chunk + col;

  bf16x8 qreg[KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk)
    qreg[kk] = head_valid ? load8(p.q + ((long)b * p.Hq + hq) * D + 32 * kk + 8 * g) : zero8();
  const float scale2 = p.scale2 * (E4M3 && p.c.ks ? p.c.ks[hkv] : 1.f);

  // table entries of the split, from its last page down: lane i holds the one i pages below
  // `top`; groups of 16 rows are walked downwards
  const int gpp = p.c.page_size / kPageRows;
  const int32_t* row = p.table + (long)b * p.W;
  int page = 0, within = 0, top = 0, entries = -1;
  const auto load_entries = [&]() {
    top = page;
    const int at = page - lane;
    entries = at >= 0 && at < p.W ? row[at] : -1;
  };
  if (t_hi > t_lo) {
    const int last = 2 * t_hi - 1;
    page = last / gpp;
    within = last - page * gpp;
    load_entries();
  }
  // byte offset of the next group below (-1: its page is outside the pool)
  const auto next_group = [&]() -> long {
    if (page < 0) return -1;
    if (top - page >= 64) load_entries();
    const int number = __builtin_amdgcn_readlane(entries, top - page);
    const long off = number * p.c.page_stride + hkv * p.c.head_stride +
                     (long)(within * kPageRows) * p.c.token_stride;
    if (within == 0) {
      within = gpp;
      --page;
    }
    --within;
    return (unsigned)number < (unsigned)p.c.num_pages ? off : -1;
  };

  const uint32_t lane_off = (uint32_t)(lane / CPR) * (uint32_t)p.c.token_stride + (lane % CPR) * 16;
  const uint32_t step = (uint32_t)(RPI * p.c.token_stride);
  typedef bf16x8 Tile[2 * IPG];          // raw bytes (16 per lane and instruction)
  // rows of group h (0, 1) of tile t that exist: of those the resource covers every byte
  const auto rows_of = [&](int t, int h, long off) {
    return off < 0 ? 0 : max(0, min(kPageRows, n - (2 * t + h) * kPageRows));
  };
  const auto load_tile = [&](const char* base, int t, long off0, long off1, Tile& x) {
    const auto r0 = make_rsrc(base + max(off0, 0l), (uint32_t)(rows_of(t, 0, off0) * p.c.token_stride));
    const auto r1 = make_rsrc(base + max(off1, 0l), (uint32_t)(rows_of(t, 1, off1) * p.c.token_stride));
#pragma unroll
    for (int i = 0; i < IPG; ++i) {
      x[i] = buf_load8_stream(r0, lane_off + i * step);
      x[IPG + i] = buf_load8_stream(r1, lane_off + i * step);
    }
  };
  bf16* mine = slot[w];
  const auto to_lds = [&](const Tile& x) {
#pragma unroll
    for (int i = 0; i < 2 * IPG; ++i) {
      const int r = i * RPI + lane / CPR, c = lane % CPR;
      if constexpr (E4M3) {
        const i32x4 raw = __builtin_bit_cast(i32x4, x[i]);
        bf16x8 lo, hi;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[j], 1.f, false);
          const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[j], 1.f, true);
          lo[4 * j] = a[0];
          lo[4 * j + 1] = a[1];
          lo[4 * j + 2] = d[0];
          lo[4 * j + 3] = d[1];
          const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[2 + j], 1.f, false);
          const bf16x2 f = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[2 + j], 1.f, true);
          hi[4 * j] = e[0];
          hi[4 * j + 1] = e[1];
          hi[4 * j + 2] = f[0];
          hi[4 * j + 3] = f[1];
        }
        store8(mine + r * LD + c * 16, lo);
        store8(mine + r * LD + c * 16 + 8, hi);
      } else {
        store8(mine + r * LD + c * 8, x[i]);
      }
    }
  };

  float m = kNegInf, l = 0.f;
  f32x4 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  int cnt = 0;
  unsigned legal = 0, vloads = 0;
  unsigned long long hsum = 0;

  for (int t = t_hi - 1; t >= t_lo; --t) {
    const long off1 = next_group(), off0 = next_group();
    const int rows0 = rows_of(t, 0, off0), rows1 = rows_of(t, 1, off1);
    if (rows0 + rows1 == 0) continue;    // no key of the tile is there
    ++legal;
    Tile x;
    load_tile(p.c.k, t, off0, off1, x);
    to_lds(x);
    load_tile(p.c.v, t, off0, off1, x);
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      s0 = mfma16(load8(mine + col * LD + 32 * kk + 8 * g), qreg[kk], s0);
      s1 = mfma16(load8(mine + (16 + col) * LD + 32 * kk + 8 * g), qreg[kk], s1);
    }
    float sv[8], mt = kNegInf;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sv[r] = 4 * g + r < rows0 ? s0[r] * scale2 : kNegInf;
      sv[4 + r] = 4 * g + r < rows1 ? s1[r] * scale2 : kNegInf;
      mt = fmaxf(mt, fmaxf(sv[r], sv[4 + r]));
    }
    mt = fmaxf(mt, __shfl_xor(mt, 16));
    mt = fmaxf(mt, __shfl_xor(mt, 32));
    const bool demand = head_valid && (l == 0.f || mt - (m + fast_log2(l)) >= thr2);
    if (!wave_any(demand)) continue;
    ++vloads;
    float alpha = 1.f, m_new = m;
    if (demand) {
      m_new = fmaxf(m, mt);
      alpha = m_new == kNegInf ? 1.f : fast_exp2(m - m_new);
    }
    const float shift = m_new == kNegInf ? 0.f : m_new;   // a tile of -inf scores adds 0
    float ps = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      sv[r] = demand ? fast_exp2(sv[r] - shift) : 0.f;
      ps += sv[r];
    }
    ps += __shfl_xor(ps, 16);
    ps += __shfl_xor(ps, 32);
    if (demand) {
      l = alpha * l + ps;
      m = m_new;
      ++cnt;
      if (p.counters) hsum += tile_hash(b, hq, 0, t);
    }
    to_lds(x);
    bf16x8 ph, pl;
    split_bf16x8(sv, ph, pl);
    const bf16x8 pr = rest_bf16x8(sv, ph, pl);
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      const bf16* vrow = mine + (4 * g + (col >> 2)) * LD + 16 * db + 4 * (col & 3);
      const bf16x8 a = cat(lds_read_tr(vrow), lds_read_tr(vrow + 16 * LD));
      acc[db] = mfma16(a, ph, acc[db] * alpha);
      acc[db] = mfma16(a, pl, acc[db]);
      if (!p.o_bf16) acc[db] = mfma16(a, pr, acc[db]);
    }
  }

  // join the wavefronts: a common reference per head, the accumulators scaled to it and added
  if (g == 0) {
    refs[w][col] = m;
    sums[w][col] = l;
    counts[w][col] = cnt;
  }
  __syncthreads();
  float M = kNegInf;
#pragma unroll
  for (int u = 0; u < kPagedWaves; ++u) M = fmaxf(M, refs[u][col]);
  if (M == kNegInf) M = 0.f;
  {
    const float f = fast_exp2(m - M);    // 0 for a wavefront without keys
    float* out = reinterpret_cast<float*>(mine);
    static_assert(sizeof(slot[0]) >= 16 * D * sizeof(float), "an accumulator fits a tile");
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      *reinterpret_cast<f32x4*>(out + (db * 64 + lane) * 4) = acc[db] * f;
  }
  __syncthreads();
  const int nb = max(1, (T + kPagedWaves * p.tps - 1) / (kPagedWaves * p.tps));
  for (int i = threadIdx.x; i < NDB * 64; i += kPagedWaves * 64) {
    const int ln = i & 63, db = i >> 6, c = ln & 15, d = 16 * db + 4 * (ln >> 4);
    if (c >= nh) continue;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float L = 0.f, mx = kNegInf;
    int kept = 0;
#pragma unroll
    for (int u = 0; u < kPagedWaves; ++u) mx = fmaxf(mx, refs[u][c]);
    const float ref = mx == kNegInf ? 0.f : mx;
#pragma unroll
    for (int u = 0; u < kPagedWaves; ++u) {
      o += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(slot[u]) + i * 4);
      L += sums[u][c] * fast_exp2(refs[u][c] - ref);
      kept += counts[u][c];
    }
    const float inv = L != 0.f ? (E4M3 && p.c.vs ? p.c.vs[hkv] : 1.f) / L : 0.f;
    const float lse = L != 0.f ? (ref + fast_log2(L)) * kLn2 : kNegInf;
    const long bh = (long)b * p.Hq + hkv * grp + 16 * chunk + c;
    if (nb == 1) {
      store_out4(p.o, bh * D + d, o * inv, p.o_bf16);
      if (d == 0) {
        p.lse[bh] = lse;
        if (p.head_tiles) p.head_tiles[bh] = kept;
      }
    } else {
      float* pp = p.part + (bh * p.nblk + blk) * (D + kDecStride);
      *reinterpret_cast<f32x4*>(pp + d) = o * inv;
      if (d == 0) {
        pp[D] = lse;
        pp[D + 1] = __int_as_float(kept);
      }
    }
  }
  if (p.counters) {
    if (head_valid && g == 0 && cnt) {
      atomicAdd(&p.counters[kCntRetained], (unsigned long long)cnt);
      atomicAdd(&p.counters[kCntSlots], (unsigned long long)cnt * kDecBk);
      atomicAdd(&p.counters[kCntSetHash], hsum);
    }
    if (lane == 0 && legal) {
      atomicAdd(&p.counters[kCntLegal], (unsigned long long)legal * nh);
      atomicAdd(&p.counters[kCntVTiles], (unsigned long long)legal);
      atomicAdd(&p.counters[kCntVNeeded], (unsigned long long)vloads);
    }
  }
}

// Joins the partials of the sequences that have more than one: one workgroup per query head.
template <int D>
__global__ __launch_bounds__(D) void mala_paged_join_kernel(PagedDecParams p) {
  __shared__ float lses[D];
  const long bh = blockIdx.x;
  const int b = (int)(bh / p.Hq), n = min(max(p.lens[b], 0), p.max_len);
  const int T = (n + kDecBk - 1) / kDecBk, per = kPagedWaves * p.tps, nb = (T + per - 1) / per;
  if (nb <= 1) return;                   // the decode kernel wrote the outputs
  const float* pp = p.part + bh * p.nblk * (D + kDecStride);
  float mx = kNegInf;
  for (int s = 0; s < nb; ++s) mx = fmaxf(mx, pp[(long)s * (D + kDecStride) + D]);
  const float ref = mx == kNegInf ? 0.f : mx;
  float z = 0.f, o = 0.f;
  int kept = 0;
  for (int s = 0; s < nb; ++s) {
    const float* x = pp + (long)s * (D + kDecStride);
    const float f = expf(x[D] - ref);    // 0 for a part without keys
    z += f;
    o += f * x[threadIdx.x];
    kept += __float_as_int(x[D + 1]);
  }
  const float inv = z != 0.f ? 1.f / z : 0.f;
  lses[threadIdx.x] = o * inv;
  __syncthreads();
  if (threadIdx.x < D / 4)
    store_out4(p.o, bh * D + 4 * threadIdx.x, *reinterpret_cast<f32x4*>(lses + 4 * threadIdx.x),
               p.o_bf16);
  if (threadIdx.x == 0) {
    p.lse[bh] = z != 0.f ? ref + logf(z) : kNegInf;
    if (p.head_tiles) p.head_tiles[bh] = kept;
  }
}

int tiles_per_wave(int split_tokens) { return split_tokens / kDecBk; }

template <int D, bool E4M3>
void launch_t(const PagedDecParams& p, hipStream_t st) {
  const long grid = (long)p.B * p.c.Hkv * p.nchunk * p.nblk;
  hipLaunchKernelGGL((mala_paged_decode_kernel<D, E4M3>), dim3((unsigned)grid),
                     dim3(kPagedWaves * 64), 0, st, p);
  if (p.nblk > 1)
    hipLaunchKernelGGL(mala_paged_join_kernel<D>, dim3((unsigned)(p.B * p.Hq)), dim3(D), 0, st, p);
}

}  // namespace

int paged_decode_blocks(int B, int Hq, int Hkv, int max_len, int split_tokens) {
  (void)B;
  (void)Hq;
  (void)Hkv;
  const int T = (max_len + kDecBk - 1) / kDecBk, per = kPagedWaves * tiles_per_wave(split_tokens);
  return (T + per - 1) / per;
}

hipError_t launch_paged_decode(PagedDecParams p, int D, int split_tokens, hipStream_t st) {
  p.tps = tiles_per_wave(split_tokens);
  p.nblk = paged_decode_blocks(p.B, p.Hq, p.c.Hkv, p.max_len, split_tokens);
  p.nchunk = (p.Hq / p.c.Hkv + 15) / 16;
  if (D == 128)
    p.c.e4m3 ? launch_t<128, true>(p, st) : launch_t<128, false>(p, st);
  else
    p.c.e4m3 ? launch_t<64, true>(p, st) : launch_t<64, false>(p, st);
  return hipGetLastError();
}

}  // namespace mala
