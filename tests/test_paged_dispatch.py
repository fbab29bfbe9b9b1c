"""How a paged decode is shared out (csrc/mala_paged_dispatch.h), on the CPU: a small C++
program compiled against the header does what the kernels do with it for random batches.
Every tile has to be some run's, in whole splits, and the blocks have to fit the grid and the
workspace that the host made for any lengths."""
import random
import shutil
import subprocess

import pytest

from paper_2609_32712_amd import build as libbuild

CXX = shutil.which("g++")
pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "mala_paged_dispatch.h"
using namespace mala;
int main() {
  int B, Hq, Hkv, D, e4m3, max_len, split, dense;
  while (std::scanf("%d %d %d %d %d %d %d %d", &B, &Hq, &Hkv, &D, &e4m3, &max_len, &split, &dense) == 8) {
    const PagedPlan x = paged_plan(B, Hq, Hkv, D, e4m3, max_len, split, dense);
    const int runs = paged_runs(x.mode);
    std::vector<int> t(B);
    unsigned total = 0;
    int longest = 0;
    for (int& n : t) {
      if (std::scanf("%d", &n) != 1) return 1;
      n = (std::min(n, max_len) + kPagedTile - 1) / kPagedTile;
      total += n;
      longest = std::max(longest, n);
    }
    const unsigned per_block = paged_block_tiles(total, longest, B, x.target, x.ragged, x.min_tpw, x.unit, runs);
    long blocks = 0;
    const char* bad = "";
    for (int n : t) {
      const int nb = paged_blocks_of(n, per_block), tpw = paged_run_tiles(n, nb, x.unit, runs);
      blocks += nb;
      if (tpw % x.unit) bad = "part of a split";
      if ((long)nb * runs * tpw < n) bad = "tiles left over";
      if (tpw > (int)(per_block / runs)) bad = "a run longer than the block's";
      if (x.blocks == B && nb > 1) bad = "a partial without a workspace";
    }
    if (blocks > x.blocks) bad = "more blocks than the grid";
    if (x.blocks > paged_decode_blocks(B, Hq, Hkv, D, max_len, split)) bad = "more than the workspace";
    // the places of a small grid: every chunk of every item once, the chunks of one on one XCD
    const long items = (long)x.blocks * Hkv;
    if (items * x.nchunk < 20000) {
      const unsigned grid = paged_grid((int)items, x.nchunk);
      if (grid > 256 && grid % 256) bad = "part of a round";
      std::vector<int> seen(items * x.nchunk), xcd(items, -1);
      for (unsigned at = 0; at < grid; ++at) {
        const int item = paged_item((int)at, x.nchunk), chunk = paged_chunk((int)at, x.nchunk);
        if (item < 0 || chunk < 0 || chunk >= x.nchunk) bad = "no such chunk";
        else if (item < items) {
          ++seen[(long)item * x.nchunk + chunk];
          if (xcd[item] >= 0 && xcd[item] != (int)(at % 8)) bad = "chunks apart";
          xcd[item] = at % 8;
        }
      }
      for (int n : seen) if (n != 1) bad = "a chunk left out or done twice";
    }
    std::printf("%d %d %ld %s.\n", x.mode, x.blocks, blocks, bad);
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    src, exe = str(d / "ask.cpp"), str(d / "ask")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I" + libbuild.CSRC, src, "-o", exe], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, list(c[:8]) + list(c[8]))) for c in cases)
        out = subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout
        got = [ln.split(" ", 3) for ln in out.splitlines()]
        assert len(got) == len(cases)
        return [(int(a), int(b), int(c), d) for a, b, c, d in got]
    return run


def _lens(rng, B, n, kind):
    if kind == "full":
        return [n] * B
    if kind == "one":
        return [n] + [rng.choice([0, 1])] * (B - 1)
    if kind == "log":
        return [int(round(2 ** rng.uniform(0, n.bit_length() - 1))) for _ in range(B)]
    return [rng.randint(0, n) for _ in range(B)]


def test_blocks_cover_every_tile_and_fit_the_grid(ask):
    rng = random.Random(5)
    cases = []
    for _ in range(4000):
        Hkv = rng.choice([1, 1, 2, 3, 8, 16, 64, 700])
        B = int(round(2 ** rng.uniform(0, 9)))
        n = int(round(2 ** rng.uniform(0, rng.choice([8, 14, 20]))))
        cases.append((B, Hkv * rng.choice([1, 4, 17, 40]), Hkv, rng.choice([64, 128]),
                      rng.choice([0, 1]), n, 32 * rng.choice([1, 2, 3, 4, 8, 16, 1000]),
                      rng.choice([0, 1]), _lens(rng, B, n, rng.choice(["full", "one", "log", "any"]))))
    for big in (2 ** 31 - 65, 1 << 30):
        for dense in (0, 1):
            cases.append((1, 8, 1, 128, 0, big, 2 ** 31 - 32, dense, [big]))
            cases.append((7, 8, 8, 64, 1, big, 64, dense, [big, 0, 5, 9999999, 1, 32, 33]))
    for c, got in zip(cases, ask(cases)):
        assert got[3] == ".", (c[:8], got)


def test_modes_of_measured_calls(ask):
    full = lambda B, n: [n] * B
    cases = [
        (1, 8, 2, 128, 0, 200, 256, 1, full(1, 200)),            # two workgroups, no join
        (1, 32, 8, 128, 0, 4096, 128, 0, full(1, 4096)),         # 256 splits: shared
        (16, 32, 8, 128, 0, 8192, 256, 0, full(16, 8192)),       # 4096 splits: a wavefront each
        (16, 32, 8, 128, 0, 131072, 256, 1, full(16, 131072)),   # a workgroup per CU: 256 of them
        (32, 32, 8, 128, 0, 2048, 256, 1, full(32, 2048)),       # a sequence per workgroup
        (1, 8, 1, 128, 0, 512, 256, 1, full(1, 512)),            # 16 tiles: one workgroup
        (1, 8, 1, 128, 0, 513, 256, 1, full(1, 513)),            # 17: joined
        (16, 32, 8, 128, 0, 768, 256, 1, full(16, 768)),         # 24, 128 workgroups: one each
        (16, 32, 8, 128, 0, 768, 128, 0, full(16, 768)),         # ... but not at tau > 0
        (32, 32, 8, 128, 0, 1024, 128, 0, full(32, 1024)),       # 32, a workgroup per CU: one each
        (32, 32, 8, 128, 0, 1025, 128, 1, full(32, 1025)),       # 33: could need a join
    ]
    got = ask(cases)
    assert [g[0] for g in got] == [0, 2, 1, 0, 0, 0, 0, 0, 1, 1, 0]
    assert [g[2] for g in got][:3] == [1, 32, 32]
    assert got[0][1] == 1 and got[3][2] * 8 <= 256 and got[4][2] == 32
    assert got[5][1] == got[5][2] == 1 and got[6][2] > 1
    assert got[7][1] == 16 and got[8][1] > 16 and got[9][1] == 32 and got[10][1] > 32
