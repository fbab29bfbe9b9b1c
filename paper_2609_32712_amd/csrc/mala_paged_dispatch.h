// How a paged decode is shared out: the host's launch rules and the arithmetic that the
// kernels share with them.  Plain C++ (the tests compile it for the CPU).
#pragma once
#include <stdint.h>

#include <algorithm>

#include "mala_dispatch.h"

#ifdef __HIP__
#define MALA_HOST_DEVICE __host__ __device__
#else
#define MALA_HOST_DEVICE
#endif

namespace mala {

constexpr int kPagedTile = 32;           // keys per decision tile
constexpr int kPagedWaves = 4;           // wavefronts of a workgroup
constexpr int kXcds = 8;                 // workgroups are dealt to the XCDs in turn

// How a block of tiles is worked on: kDense (tau = 0) and kChain, a run of tiles per wavefront
// (kChain: of whole splits, tested one after the other); kTeam, whole splits by all
// wavefronts, a tile each at a time.
enum { kDense = 0, kChain = 1, kTeam = 2 };
constexpr int paged_runs(int mode) { return mode == kTeam ? 1 : kPagedWaves; }   // per block

// Tiles per block of a batch of B sequences, `total` tiles in all and `longest` in one, whole
// units per run.  Where the longest is over 5 / 4 of the average, blocks are smaller: they can be
// dealt more evenly.  (A floor plus one is at least the even share, so that at most target + B
// blocks come of it.)
MALA_HOST_DEVICE inline unsigned paged_block_tiles(unsigned total, int longest, int B, int target,
                                                   int ragged, int min_tpw, unsigned unit, int runs) {
  const int blocks = (float)longest * B > 1.25f * total ? ragged : target;
  const unsigned even = total / ((unsigned)blocks * runs) + 1;
  const unsigned tpw = even > (unsigned)min_tpw ? even : (unsigned)min_tpw;
  return runs * (unit == 1 ? tpw : (tpw + unit - 1) / unit * unit);
}
// Blocks of a sequence of t tiles, and tiles per run of it: even runs, whole units.
MALA_HOST_DEVICE inline int paged_blocks_of(int t, unsigned per_block) {
  const int n = (int)((t + per_block - 1) / per_block);
  return n > 1 ? n : 1;
}
MALA_HOST_DEVICE inline int paged_run_tiles(int t, int blocks, unsigned unit, int runs) {
  const unsigned n = ((unsigned)t + blocks * runs - 1) / (unsigned)(blocks * runs);
  return (int)(unit == 1 ? n : (n + unit - 1) / unit * unit);
}

// Blocks are dealt in classes of sizes, the largest class (7) first: of `tpw` tiles per run of `runs`, or of
// `tpw` in all of one, at most per_block / runs.  (By the tiles of each block, since a sequence's last one
// is often small.  us per call by the run length / by the tiles, 8 bits: 64 caches of up to 4000 tokens
// at tau > 0 58.7 / 52.6, 32 of up to 30000 195 / 184, 64 log-uniform ones of up to 16384 at tau = 0 42.1 /
// 40.7, 48 of up to 8192 70.0 / 71.2.  These are single draws: with other lengths 32 of up to 30000 lose up
// to 4%, and 32 of up to 4000 at tau = 0, D = 64, 1 to 5%.)
constexpr int kPagedClasses = 8;
MALA_HOST_DEVICE inline int paged_run_class(int tpw, unsigned per_block, int runs) {
  const int c = (int)(tpw * (unsigned)kPagedClasses / (per_block / runs + 1u));
  return c < kPagedClasses - 1 ? c : kPagedClasses - 1;
}

// The rule's test of a tile with the largest score mt (base 2) against its split's log-sum `run`, and
// the early one, with the log-sum before the tile above has been added: what the first would
// retain the second must not rule out.  A log-sum only grows, but as an fp32: adding a tile can
// take it down by the rounding of the sum (1e-5 at most) and where that crosses a step of fp32
// by the step, 2^-23 |run|.  The margin covers both, and the differences' own rounding.
MALA_HOST_DEVICE inline bool paged_retains(float mt, float run, float thr2) {
#ifdef __clang__
#pragma clang fp contract(off)
#endif
  return mt - run >= thr2;
}
MALA_HOST_DEVICE inline bool paged_may_retain(float mt, float run, float thr2) {
#ifdef __clang__
#pragma clang fp contract(off)
#endif
  return mt - run >= thr2 - __builtin_fmaf(__builtin_fabsf(run), 0x1p-21f, 1e-2f);
}

// Where a KV head has more than 16 query heads, its chunks of 16 read the same K and V: workgroups
// kXcds places apart run on one XCD and share its L2 (16 x 8192 tokens, 64 heads on 2, when it was
// taken: 50.6 us with the chunks next to each other, 35.4 so; 36.5 now, with a third term of P).
// The item (block of a sequence, KV head) and the chunk at a place:
MALA_HOST_DEVICE inline int paged_item(int place, int nchunk) {
  return nchunk == 1 ? place : place / kXcds / nchunk * kXcds + place % kXcds;
}
MALA_HOST_DEVICE inline int paged_chunk(int place, int nchunk) {
  return nchunk == 1 ? 0 : place / kXcds % nchunk;
}
// Places that cover all chunks of the items; whole rounds of the CUs where there are several, since
// every other round is dealt backwards.
inline unsigned paged_grid(int items, int nchunk) {
  const unsigned n = nchunk == 1 ? items : ((unsigned)items + kXcds - 1) / kXcds * kXcds * nchunk;
  return n > (unsigned)kNumCus ? (n + kNumCus - 1) / kNumCus * kNumCus : n;
}

// Workgroups that a large call is shared out to.  A CU gets its own share of HBM's rate, so it is
// the CU with the most tiles that sets the time: equal workgroups should be as many as there are
// CUs, or a multiple.  With tiles of 16 KB (K and V of 32 bf16 rows of 128) the four wavefronts
// of one workgroup keep 64 KB on their way, which is enough; smaller tiles need more of them.
// us per call with 256 / 336-512 / 608-1024 workgroups: 16 ragged 8192-token caches 52.6 / 63.5 /
// 58.4, 32 x 2048 tokens 47.0 / 50.4 / 50.4, one of 32768 28.9 / 31 / 32; of 8 KB tiles, 64
// ragged e4m3 caches 49.4 / 45.6 / 45.2; of 4 KB, 32 ragged ones (D = 64) 25.6 / 20.6 / 20.7.
inline int paged_target_groups(int D, bool e4m3) { return kNumCus * (128 / D) * (e4m3 ? 2 : 1); }

// And of sequences of unequal length (tau = 0), dealt by their sizes, twice as many: 16 ragged
// 8192-token caches 57.3 / 52.1, 64 log-uniform ones of up to 32768 127.5 / 124.0, 128 of up to 2048
// 92.3 / 91.2.  (With tau > 0 blocks are whole splits, and the next smaller ones a third too small.)
constexpr int kRaggedGroups = 2 * kNumCus;

// Caches of up to so many tiles stay in one workgroup each, without a join: a tile more takes a
// wavefront 1.2 us (0.8 at D = 64), the join 2.5 behind its launch.  Few workgroups leave CUs free
// that the blocks of a split cache could use: 16 tiles; where workgroups are as many as half the
// CUs 24 (tau = 0), as many as the CUs 32.  us per call in blocks / whole (8 KV heads, D = 128): one
// cache of 512 tokens 7.9 / 7.9, of 768 8.0 / 9.7; 8 of 768 11.0 / 12.3; 16 of 768 14.4 / 13.4 (tau > 0
// 15.6 / 17.1), of 1024 17.0 / 16.4, of 0..1024 14.6 / 15.3; 32 of 1024 26.0 / 23.8 (27.1 / 25.3), of
// 0..1024 19.5 / 17.8 (21.4 / 18.1), log-uniform 11.2 / 12.0; 64 of 0..768 26.5 / 20.3; 128 e4m3 ones (D =
// 64) of 0..1024 25.1 / 17.3.  64 tiles: 64 of 0..2048 52.8 / 48.6, but log-uniform 21.5 / 28.3.
inline int paged_single_tiles(long groups, bool dense) {
  return groups >= kNumCus ? 32 : dense && groups >= kNumCus / 2 ? 24 : 16;
}

// tau > 0: splits up to which the wavefronts of a workgroup share them.  us per call, a wavefront
// per split / shared: one cache of 1000 tokens (64 splits of 128) 13.1 / 9.6, of 4096 (256) 14.2 /
// 11.9, 4096 in splits of 256 18.9 / 12.9, 32768 in splits of 512 (512 of them) 32.0 / 31.0; from
// 1024 splits on no gain, and a wavefront per split fetches only the V tiles it needs.
constexpr long kTeamSplits = 512;

struct PagedPlan {
  int target, ragged;   // blocks per KV head and chunk that a call is shared out to, if ragged
  int unit;             // tiles per split (tau = 0: 1)
  int min_tpw;          // tiles per run at least
  int blocks;           // of all sequences at most
  int mode, nchunk;
};
inline PagedPlan paged_plan(int B, int Hq, int Hkv, int D, bool e4m3, int max_len,
                            int split_tokens, bool dense) {
  const int T = (max_len + kPagedTile - 1) / kPagedTile;
  PagedPlan x;
  const int nchunk = x.nchunk = (Hq / Hkv + 15) / 16;
  x.unit = dense ? 1 : split_tokens / kPagedTile;
  const long splits = (long)B * Hkv * nchunk * ((T + x.unit - 1) / x.unit);
  x.mode = dense ? kDense : x.unit > 1 && splits <= kTeamSplits ? kTeam : kChain;
  const int runs = paged_runs(x.mode);
  x.target = (int)std::max<long>(1, (x.mode == kTeam ? kTeamSplits
                                                             : paged_target_groups(D, e4m3)) /
                                       (Hkv * nchunk));
  x.ragged = x.mode == kDense ? std::max(x.target, kRaggedGroups / (Hkv * nchunk)) : x.target;
  x.min_tpw = T <= paged_single_tiles((long)B * Hkv * nchunk, dense) ? (T + runs - 1) / runs : 1;
  const long tpw = (x.min_tpw + x.unit - 1) / x.unit * (long)x.unit;
  const long most = (T + runs * tpw - 1) / (runs * tpw);
  x.blocks = (int)std::min<long>({(long)B + x.ragged, B * most, (long)INT32_MAX});
  return x;
}

// The longest cache whose tiles and rows can be counted in 32 bits.
constexpr int kPagedMaxLen = INT32_MAX - 64;

// Blocks of all sequences at most, whatever the type and tolerance (the workspace holds their
// partials).
inline int paged_decode_blocks(int B, int Hq, int Hkv, int D, int max_len, int split_tokens) {
  int n = 0;
  for (int i = 0; i < 4; ++i)
    n = std::max(n, paged_plan(B, Hq, Hkv, D, i & 1, max_len, split_tokens, i & 2).blocks);
  return n;
}

}  // namespace mala
