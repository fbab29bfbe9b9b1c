"""The order in which the blocks of a ragged paged decode are dealt (CPU): the kernel gives the
longest runs of up to 64 sequences the first places, in eight classes of run lengths.  Every
place has to be one block's, and the blocks of a sequence have to keep the numbers under which
the join looks for them."""
import random
import shutil
import subprocess

import pytest

from paper_2609_32712_amd import build as libbuild

CXX = shutil.which("g++")
pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")

# what share_of does by lanes, in loops
PROGRAM = r"""
#include <cstdio>
#include <map>
#include <set>
#include <vector>
#include "mala_paged_dispatch.h"
using namespace mala;
int main() {
  int B, Hq, Hkv, D, e4m3, max_len, split, dense;
  while (std::scanf("%d %d %d %d %d %d %d %d", &B, &Hq, &Hkv, &D, &e4m3, &max_len, &split, &dense) == 8) {
    const PagedPlan x = paged_plan(B, Hq, Hkv, D, e4m3, max_len, split, dense);
    const int W = paged_runs(x.mode);
    std::vector<int> t(B);
    unsigned total = 0;
    int longest = 0;
    for (int& n : t) {
      if (std::scanf("%d", &n) != 1) return 1;
      n = (std::min(n, max_len) + kPagedTile - 1) / kPagedTile;
      total += n;
      longest = std::max(longest, n);
    }
    const unsigned per_block = paged_block_tiles(total, longest, B, x.target, x.ragged, x.min_tpw, x.unit, W);
    const char* bad = "";
    int sorted_parts = 0, before = 0;
    std::vector<std::vector<int>> covered(B);
    for (int b = 0; b < B; ++b) covered[b].assign(t[b], 0);
    for (int b0 = 0; b0 < B; b0 += 64) {
      const int here = std::min(64, B - b0);
      std::vector<int> nb(here), tpw(here), end(here), from(here);
      int all = 0;
      bool sort = false;
      for (int i = 0; i < here; ++i) {
        nb[i] = paged_blocks_of(t[b0 + i], per_block);
        tpw[i] = paged_run_tiles(t[b0 + i], nb[i], x.unit, W);
        all += nb[i];
        end[i] = all;
        from[i] = end[i] - nb[i];
        sort |= tpw[i] > 4;
      }
      if (sort) {
        ++sorted_parts;
        int base = 0;
        for (int c = kPagedClasses - 1; c >= 0; --c)
          for (int i = 0; i < here; ++i)
            if (paged_run_class(tpw[i], per_block, W) == c) {
              from[i] = base;
              base += nb[i];
            }
        if (base != all) bad = "a class outside the eight";
      }
      std::vector<int> taken(all, -1);
      int last_class = kPagedClasses;
      for (int place = 0; place < all; ++place) {
        int who = -1;
        for (int i = 0; i < here; ++i)
          if (from[i] <= place && place < from[i] + nb[i]) {
            if (who >= 0) bad = "two blocks at one place";
            who = i;
          }
        if (who < 0) { bad = "no block at a place"; continue; }
        if (sort) {
          const int c = paged_run_class(tpw[who], per_block, W);
          if (c > last_class) bad = "a longer run behind a shorter one's class";
          last_class = c;
        }
        const int first = before + end[who] - nb[who], blk = place - from[who];
        if (blk < 0 || blk >= nb[who] || first < before || first + blk >= before + all) bad = "a number that is not the sequence's";
        else if (taken[first + blk - before] >= 0) bad = "one number for two blocks";
        else taken[first + blk - before] = who;
        for (int w = 0; w < W; ++w) {
          const int lo = std::min(t[b0 + who], (blk * W + w) * tpw[who]), hi = std::min(t[b0 + who], lo + tpw[who]);
          for (int k = lo; k < hi; ++k) ++covered[b0 + who][k];
        }
      }
      before += all;
    }
    for (auto& c : covered)
      for (int n : c)
        if (n != 1) bad = "a tile left out or worked on twice";
    if (before > x.blocks) bad = "more blocks than places";
    int runs = 0, cut = 0;
    for (int n : t) {
      const int nb = paged_blocks_of(n, per_block);
      runs = std::max(runs, paged_run_tiles(n, nb, x.unit, W));
      cut = std::max(cut, nb);
    }
    const bool dealt = B > 1 && (long)x.blocks * Hkv * x.nchunk > kNumCus;
    std::printf("%d %d %d %d %d %d %s.\n", sorted_parts, before, x.mode, runs, cut, (int)dealt, bad);
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("order")
    src, exe = str(d / "ask.cpp"), str(d / "ask")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I" + libbuild.CSRC, src, "-o", exe], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, list(c[:8]) + list(c[8]))) for c in cases)
        out = subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout
        got = [ln.split(" ", 6) for ln in out.splitlines()]
        assert len(got) == len(cases)
        return [dict(zip(("sorted", "blocks", "mode", "run", "cut", "dealt"), map(int, g[:6])), bad=g[6])
                for g in got]
    return run


def test_every_place_is_one_block_and_every_tile_one_run(ask):
    rng = random.Random(7)
    cases = []
    for _ in range(600):
        Hkv = rng.choice([1, 2, 8, 16, 64])
        B = int(round(2 ** rng.uniform(0, 8.5)))
        n = int(round(2 ** rng.uniform(5, 15)))
        kind = rng.choice(["any", "log", "one"])
        lens = [rng.randint(0, n) if kind == "any" else int(2 ** rng.uniform(0, n.bit_length() - 1)) if kind == "log"
                else rng.choice([0, 1, 40]) for _ in range(B)]
        lens[rng.randrange(B)] = n
        cases.append((B, Hkv * rng.choice([1, 4, 17, 40]), Hkv, rng.choice([64, 128]), rng.choice([0, 1]),
                      n, 32 * rng.choice([1, 2, 4, 8, 16, 64]), rng.choice([0, 1]), lens))
    got = ask(cases)
    for c, g in zip(cases, got):
        assert g["bad"] == ".", (c[:8], g)
    assert sum(g["sorted"] > 0 for g in got) > 100
    assert sum(g["sorted"] > 0 and g["cut"] > 2 for g in got) > 50


# the calls of test_paged_long.py, and the branches of the kernels they are there for
def test_long_calls_reach_their_branches(ask):
    from test_paged_long import CALLS
    got = ask([(len(c["lens"]), c["Hq"], c["Hkv"], c["D"], int(c["e4m3"]), max(c["lens"]), c["split"],
                int(c["tau"] == 0), c["lens"]) for c in CALLS.values()])
    for (name, c), g in zip(CALLS.items(), got):
        assert g["bad"] == "." and g["mode"] == c["mode"] and g["dealt"] == c["dealt"], name
        # a wavefront looks up the pages of 32 tiles at a time
        assert g["run"] > 32 if c["long"] else g["run"] > 4, (name, g)
        assert g["cut"] >= c["cut"] and g["sorted"] > 0, (name, g)
