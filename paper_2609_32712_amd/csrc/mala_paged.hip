// The paged KV cache around the decode: page tables from lengths, rows into pages, pages
// back to packed rows (gfx950).
//
// Position p of request r lives in slot table[r][p / P] P + p mod P, P rows per page.
#include "mala_device.h"
#include "mala_paged.h"

namespace mala {

namespace {

// Data that a call moves once: past the caches' retention.  (e4m3 rows are read by the write
// as two halves of 32 bytes per lane, which an ordinary load keeps close for the second.)
template <class T>
__device__ __forceinline__ T load_once(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const T*>(p));
}
template <class T>
__device__ __forceinline__ void store_once(void* p, T v) {
  __builtin_nontemporal_store(v, reinterpret_cast<T*>(p));
}

// ------------------------------------------------------------------ page tables
// One launch: every workgroup scans the lengths of all requests (they are few: R lengths are
// 8 R bytes from the L2), so none waits for another, and then does its own share of the
// tokens and of the pages given back.  What bounds a call is latency: the loads of the
// lengths, the scan and one dependent load per token (its table entry or its page of the
// ring).  Requests that grow by a few tokens (decodes) take them by a thread each, with the
// table entry loaded before the scan; the tokens of longer ones are shared out by token.
// Inputs and outputs never share an address: a request either takes pages or gives some
// back, and the ring's popped and pushed places are disjoint while free and used pages
// together fit it.  us per call: 64 decodes 2.9 (6.6 by token, scanned by shuffles), a mix of
// 512 requests and 232000 tokens 6.2 (10.3; 9.5 with the scans by shuffles).
constexpr int kUpdFew = 4;        // tokens that a request's thread takes itself
constexpr int kUpdChunk = 1024;   // tokens (or pages given back) a workgroup takes at a time

struct Scan3 {
  int grow, need, back, many;     // many: whether some request is no thread's own
};

// Inclusive scan over the workgroup's threads; `sum` is the total.
template <int NT>
__device__ __forceinline__ Scan3 scan_block(Scan3 x, Scan3* wave_sums, Scan3* sum) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int many = __builtin_amdgcn_ballot_w64(x.many) != 0;
  x.grow = wave_scan(x.grow);
  x.need = wave_scan(x.need);
  x.back = wave_scan(x.back);
  __syncthreads();   // wave_sums of the block before have been read
  if (lane == 63) wave_sums[w] = Scan3{x.grow, x.need, x.back, many};
  __syncthreads();
  const Scan3 y = lane < NT / 64 ? wave_sums[lane] : Scan3{0, 0, 0, 0};
  const int grow = wave_scan(y.grow), need = wave_scan(y.need), back = wave_scan(y.back);
  if (w) {
    x.grow += __builtin_amdgcn_readlane(grow, w - 1);
    x.need += __builtin_amdgcn_readlane(need, w - 1);
    x.back += __builtin_amdgcn_readlane(back, w - 1);
  }
  *sum = Scan3{__builtin_amdgcn_readlane(grow, 63), __builtin_amdgcn_readlane(need, 63),
               __builtin_amdgcn_readlane(back, 63), __builtin_amdgcn_ballot_w64(y.many) != 0};
  return x;
}

// The last of the first n entries of a (ascending) that is <= x; a[0] <= x.
__device__ __forceinline__ int last_not_above(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <int NT>
__global__ __launch_bounds__(NT) void mala_paged_update_kernel(PagedUpdateParams p) {
  // the requests of the block being worked on
  __shared__ int s_start[NT], s_old[NT], s_have[NT];
  __shared__ int s_page[NT];             // its first page in the order of the ring, or -1: refused
  __shared__ int s_back[NT], s_want[NT];
  __shared__ Scan3 wave_sums[NT / 64];
  __shared__ int s_refused;

  // the last workgroup, where there are several, has no share of the chunks: it starts with the
  // requests that take their tokens by a thread each
  const int tid = threadIdx.x, G = gridDim.x > 1 ? gridDim.x - 1 : 1;
  const unsigned P = p.P;
  const int most = p.W * p.P;            // tokens a table row can hold (below 2^31 in all)
  const int head = min(max(p.state[0], 0), p.C - 1), count = min(max(p.state[1], 0), p.C);
  if (tid == 0) s_refused = 0;
  // the first of this workgroup's chunks (every G-th) that ends behind item x
  const auto my_chunk = [&](int x) {
    if ((int)blockIdx.x >= G) return INT32_MAX;
    const int c = x / kUpdChunk, over = c % G;
    return c - over + (int)blockIdx.x + ((int)blockIdx.x < over ? G : 0);
  };
  // place i < C places behind place `at` < C of the ring
  const auto ring_at = [&](unsigned at, int i) {
    at += i;
    return at >= (unsigned)p.C ? at - p.C : at;
  };
  // slot and position of a token whose page has this number
  const auto put_token = [&](int t, int number, unsigned off, int pos) {
    if (t >= p.max_tokens) return;
    p.slots[t] = (unsigned)number < (unsigned)p.num_pages ? number * p.P + (int)off : -1;
    if (p.positions) p.positions[t] = pos;
  };

  int tokens = 0, pages = 0, back = 0, taken = 0;   // of the requests before this block
                                                    // (taken: by this wavefront's, at last)
  for (int r0 = 0; r0 < p.R; r0 += NT) {
    const int r = r0 + tid, nr = min(NT, p.R - r0);
    int old = 0, now = 0;
    if (r < p.R) {
      old = min(max(p.lens[r], 0), most);
      now = min(max(p.new_lens[r], 0), most);
    }
    const int have = (old + P - 1) / P, want = (now + P - 1) / P;
    const Scan3 mine = {max(now - old, 0), max(want - have, 0), max(have - want, 0),
                        now - old > kUpdFew};
    const bool owner = (r0 / NT) % gridDim.x == gridDim.x - 1 - blockIdx.x, few = mine.grow > 0 && !mine.many;
    int entry = -1;                      // of the page that the request's next token goes on
    if (owner && few && have * (int)P > old) entry = p.table[(long)r * p.W + have - 1];
    Scan3 sum;
    const Scan3 end = scan_block<NT>(mine, wave_sums, &sum);
    const bool granted = mine.need == 0 || pages + end.need <= count;
    const int start = tokens + end.grow - mine.grow, first = pages + end.need - mine.need;
    if (owner && few) {
      for (int j = 0; j < mine.grow; ++j) {
        const int pos = old + j, page = pos / P, off = pos - page * P;
        if (page >= have) {
          entry = granted ? p.ring[ring_at(head, first + page - have)] : -1;
          if (granted && off == 0) p.table[(long)r * p.W + page] = entry;
        }
        put_token(start + j, granted ? entry : -1, off, pos);
      }
    }
    if (blockIdx.x == 0 && r < p.R) {
      p.cu[r] = start;
      p.lens_out[r] = granted ? now : old;
      if (!granted) atomicAdd(&s_refused, 1);
    }
    // pages taken up to the last granted request that needs some
    const unsigned long long takers = __builtin_amdgcn_ballot_w64(granted && mine.need);
    if (takers)
      taken = pages + __builtin_amdgcn_readlane(end.need, 63 - __builtin_clzll(takers));
    if (sum.many || sum.back) {
      s_start[tid] = start;
      s_old[tid] = old;
      s_have[tid] = have;
      s_page[tid] = granted ? first : -1;
      s_back[tid] = back + end.back - mine.back;
      s_want[tid] = mine.grow <= kUpdFew ? want : -1;    // (of a growing request: taken already?)
      __syncthreads();
      // tokens: chunks of kUpdChunk, every G-th of them this workgroup's
      const int tok_end = tokens + sum.grow;
      for (int c = my_chunk(tokens); sum.many && (long)c * kUpdChunk < tok_end; c += G) {
        const int t1 = (int)min((long)tok_end, (long)(c + 1) * kUpdChunk);
        for (int t = max(tokens, c * kUpdChunk) + tid; t < t1; t += NT) {
          const int i = last_not_above(s_start, nr, t);
          if (s_want[i] >= 0) continue;
          const int pos = s_old[i] + t - s_start[i], page = pos / P, off = pos - page * P;
          int32_t* at = p.table + (long)(r0 + i) * p.W + page;
          int number = -1;
          if (s_page[i] >= 0) {
            if (page >= s_have[i]) {
              number = p.ring[ring_at(head, s_page[i] + page - s_have[i])];
              if (off == 0) *at = number;
            } else {
              number = *at;
            }
          }
          put_token(t, number, off, pos);
        }
      }
      // pages given back, to the end of the ring
      const int back_end = back + sum.back;
      for (int c = my_chunk(back); (long)c * kUpdChunk < back_end; c += G) {
        const int j1 = (int)min((long)back_end, (long)(c + 1) * kUpdChunk);
        for (int j = max(back, c * kUpdChunk) + tid; j < j1; j += NT) {
          const int i = last_not_above(s_back, nr, j);
          const int page = s_want[i] + j - s_back[i];
          if (j < p.C - count)           // (always, while free and used pages fit the ring)
            p.ring[ring_at(head, count + j)] = p.table[(long)(r0 + i) * p.W + page];
        }
      }
      __syncthreads();                   // the block's requests have been read
    }
    tokens += sum.grow;
    pages += sum.need;
    back += sum.back;
  }
  // padding behind the last token
  for (int c = my_chunk(tokens); (long)c * kUpdChunk < p.max_tokens; c += G) {
    const int t1 = (int)min((long)p.max_tokens, (long)(c + 1) * kUpdChunk);
    for (int t = max(tokens, c * kUpdChunk) + tid; t < t1; t += NT) {
      p.slots[t] = -1;
      if (p.positions) p.positions[t] = 0;
    }
  }
  if (blockIdx.x == 0) {
    __syncthreads();                     // wave_sums of the last block have been read
    if ((tid & 63) == 0) wave_sums[tid >> 6].need = taken;
    __syncthreads();
    if (tid == 0) {
      int all = 0;
      for (int u = 0; u < NT / 64; ++u) all = max(all, wave_sums[u].need);
      p.cu[p.R] = tokens;
      p.state_out[0] = (int)ring_at(head, all);
      p.state_out[1] = count - all + min(back, p.C - count);
      p.state_out[2] = s_refused;
      p.state_out[3] = tokens;
    }
  }
}

// ------------------------------------------------------------------ rows into pages
// A thread moves 16 bytes of a row of the cache, of K and of V; a workgroup stays with a head.
// HBM-bound.
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void mala_paged_write_kernel(PagedWriteParams p) {
  constexpr int EPC = E4M3 ? 16 : 8;     // values per 16 bytes of the cache
  constexpr int CPR = D / EPC;
  const long i = (long)blockIdx.x * 256 + threadIdx.x, t = i / CPR;
  const int c = (int)(i % CPR);
  if (t >= p.T) return;
  const int slot = p.slots[t];
  const unsigned P = p.c.page_size;
  if (slot < 0 || (unsigned)slot >= p.c.num_pages * P) return;
  const unsigned page = slot / P, row = slot - page * P;
  for (int h = blockIdx.y; h < p.c.Hkv; h += gridDim.y) {
    const long src = t * p.token_stride + h * p.head_stride + c * EPC * 2;
    const long dst = page * p.c.page_stride + h * p.c.head_stride + row * p.c.token_stride + c * 16;
    if constexpr (E4M3) {
      const auto put = [&](char* pool, const char* in, float s) {
        i32x4 out;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bf16x8 x = *reinterpret_cast<const bf16x8*>(in + src + 16 * e);
          out[2 * e] = to_e4m3x4((float)x[0] / s, (float)x[1] / s, (float)x[2] / s, (float)x[3] / s);
          out[2 * e + 1] = to_e4m3x4((float)x[4] / s, (float)x[5] / s, (float)x[6] / s, (float)x[7] / s);
        }
        store_once(pool + dst, out);
      };
      put(p.c.k, p.k, p.c.ks ? p.c.ks[h] : 1.f);
      put(p.c.v, p.v, p.c.vs ? p.c.vs[h] : 1.f);
    } else {
      const i32x4 a = load_once<i32x4>(p.k + src), b = load_once<i32x4>(p.v + src);
      store_once(p.c.k + dst, a);
      store_once(p.c.v + dst, b);
    }
  }
}

// ------------------------------------------------------------------ pages to packed rows
// A workgroup takes ROWS consecutive packed rows (of every head).  HBM-bound.  Rows of bytes are read
// 8 at a time, half lines, by ordinary loads: past the caches each half fetched its line again (10 caches
// of up to 10000 rows, 8 heads, 62.4 / 59.9 us; 32 of up to 8000, 2 heads, 41.2 / 29.8).
template <int D, int FMT, int ROWS>
__global__ __launch_bounds__(256) void mala_paged_read_kernel(PagedReadParams p) {
  constexpr int CPR = D / 8;             // pieces of 8 values per row
  __shared__ int s_seq;
  const int tid = threadIdx.x, row0 = blockIdx.x * ROWS, Hkv = p.c.Hkv;
  const unsigned P = p.c.page_size;
  if (tid == 0) s_seq = 0;
  __syncthreads();
  int before = 0;                        // sequences that start at or before row0
  for (int b = tid; b < p.S; b += 256) before += p.cu[b] <= row0;
  if (before) atomicAdd(&s_seq, before);
  __syncthreads();
  const int seq0 = max(s_seq - 1, 0);
  // a thread keeps its piece of the row and its row, and goes on by heads
  constexpr int HEADS = 256 / (CPR * ROWS);   // heads at a time
  const int c = tid % CPR, row = row0 + tid / CPR % ROWS;
  int b = seq0;
  while (b < p.S && p.cu[b + 1] <= row) ++b;
  if (b >= p.S || row >= p.total) return;
  const int pos = row - p.cu[b];
  if (pos < 0 || pos >= p.max_len) return;
  const unsigned page = pos / P, off = pos - page * P;
  const int number = p.table[(long)b * p.W + page];
  const bool there = (unsigned)number < (unsigned)p.c.num_pages;
  const long at = there ? (long)number * p.c.page_stride + off * p.c.token_stride : 0;
#pragma unroll 4
  for (int h = tid / (CPR * ROWS); h < Hkv; h += HEADS) {
    const long dst = (((long)h * p.total + row) * D + c * 8) * 2;
    if constexpr (FMT != kCacheBf16) {
      const long src = at + h * p.c.head_stride + c * 8;
      i32x2 a = {0, 0}, v = a;
      if (there) {
        a = *reinterpret_cast<const i32x2*>(p.c.k + src);
        v = *reinterpret_cast<const i32x2*>(p.c.v + src);
      }
      const auto put = [&](char* out, const i32x2& x, float s) {
        i32x4 y;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (FMT == kCacheBlock) {      // (by a power of two: exact)
            y[2 * j] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[j], s, false));
            y[2 * j + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[j], s, true));
          } else {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(x[j], false);
            const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(x[j], true);
            y[2 * j] = __builtin_bit_cast(int, bf16x2{(bf16)(lo[0] * s), (bf16)(lo[1] * s)});
            y[2 * j + 1] = __builtin_bit_cast(int, bf16x2{(bf16)(hi[0] * s), (bf16)(hi[1] * s)});
          }
        }
        store_once(out + dst, y);
      };
      float ks = 1.f, vs = 1.f;
      if constexpr (FMT == kCacheBlock) {
        const unsigned blocks = P / kPageRows;
        const int64_t b = there ? ((int64_t)number * Hkv + h) * blocks + off / kPageRows : 0;
        ks = __uint_as_float(block_scale_bits(p.c.kb[b]));
        vs = __uint_as_float(block_scale_bits(p.c.vb[b]));
      } else {
        if (p.c.ks) ks = p.c.ks[h];
        if (p.c.vs) vs = p.c.vs[h];
      }
      put(p.k, a, ks);
      put(p.v, v, vs);
    } else {
      const long src = at + h * p.c.head_stride + c * 16;
      i32x4 a = {0, 0, 0, 0}, v = a;
      if (there) {
        a = load_once<i32x4>(p.c.k + src);
        v = load_once<i32x4>(p.c.v + src);
      }
      store_once(p.k + dst, a);
      store_once(p.v + dst, v);
    }
  }
}

}  // namespace

hipError_t launch_paged_update(const PagedUpdateParams& p, hipStream_t st) {
  const long chunks = ((long)p.max_tokens + kUpdChunk - 1) / kUpdChunk;
  const unsigned grid = (unsigned)(chunks <= 1 ? 1 : chunks > 256 ? 257 : chunks + 1);
  // few requests and tokens: fewer wavefronts to wait for at the barriers
  if (p.R <= 256 && chunks <= 4)
    hipLaunchKernelGGL(mala_paged_update_kernel<256>, dim3(grid), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(mala_paged_update_kernel<1024>, dim3(grid), dim3(1024), 0, st, p);
  return hipGetLastError();
}

template <int D, bool E4M3>
static void launch_write_t(const PagedWriteParams& p, hipStream_t st) {
  const long n = (long)p.T * (D / (E4M3 ? 16 : 8));
  const dim3 grid((unsigned)((n + 255) / 256), (unsigned)std::min(p.c.Hkv, 65535));
  hipLaunchKernelGGL((mala_paged_write_kernel<D, E4M3>), grid, dim3(256), 0, st, p);
}

hipError_t launch_paged_write(const PagedWriteParams& p, int D, hipStream_t st) {
  if (p.c.fmt == kCacheBlock) return launch_paged_block_write(p, D, st);
  const bool e4m3 = p.c.fmt == kCacheE4M3;
  if (D == 128)
    e4m3 ? launch_write_t<128, true>(p, st) : launch_write_t<128, false>(p, st);
  else
    e4m3 ? launch_write_t<64, true>(p, st) : launch_write_t<64, false>(p, st);
  return hipGetLastError();
}

template <int D, int FMT, int ROWS>
static void launch_read_r(const PagedReadParams& p, hipStream_t st) {
  const unsigned grid = (unsigned)(((long)p.total + ROWS - 1) / ROWS);
  hipLaunchKernelGGL((mala_paged_read_kernel<D, FMT, ROWS>), dim3(grid), dim3(256), 0, st, p);
}
// Rows of a workgroup: eight of a large batch, and where the threads of four would be more than there
// are heads for.  us per call of four / eight: 2000 rows of 8 heads 3.8 / 4.4, 8000 9.9 / 9.9, 10 caches
// of up to 10000 62.4 / 59.9, 32 of up to 8000 with 2 heads 42.1 / 29.8.
template <int D, int FMT>
static void launch_read_t(const PagedReadParams& p, hipStream_t st) {
  if (FMT != kCacheBf16 && (p.total >= 16384 || p.c.Hkv * (D / 8) < 64))
    launch_read_r<D, FMT, FMT == kCacheBf16 ? 4 : 8>(p, st);
  else
    launch_read_r<D, FMT, 4>(p, st);
}
template <int D>
static void launch_read_d(const PagedReadParams& p, hipStream_t st) {
  if (p.c.fmt == kCacheBlock)
    launch_read_t<D, kCacheBlock>(p, st);
  else if (p.c.fmt == kCacheE4M3)
    launch_read_t<D, kCacheE4M3>(p, st);
  else
    launch_read_t<D, kCacheBf16>(p, st);
}

hipError_t launch_paged_read(const PagedReadParams& p, int D, hipStream_t st) {
  D == 128 ? launch_read_d<128>(p, st) : launch_read_d<64>(p, st);
  return hipGetLastError();
}

}  // namespace mala
