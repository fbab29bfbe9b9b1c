"""The places that the blocks of a ragged paged decode are dealt to (CPU): the kernel gives the blocks of
the most tiles the first places, in eight classes, a sequence's last block by what is left for it.
Every place has to be one block's, every block has a place, and no class stands before a larger one."""
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
    int sorted = 0, small = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
      const int here = std::min(64, B - b0);
      std::vector<int> nb(here), tpw(here), from(here), last(here);
      int all = 0;
      bool sort = false;
      for (int i = 0; i < here; ++i) {
        nb[i] = paged_blocks_of(t[b0 + i], per_block);
        tpw[i] = paged_run_tiles(t[b0 + i], nb[i], x.unit, W);
        from[i] = all;
        all += nb[i];
        last[i] = all - 1;
        sort |= tpw[i] > 4;
      }
      const auto rest = [&](int i) { return t[b0 + i] - (nb[i] - 1) * W * tpw[i]; };
      const auto cls = [&](int tiles) { return paged_run_class(tiles, per_block, 1); };
      if (sort) {
        ++sorted;
        int base = 0;
        for (int c = kPagedClasses - 1; c >= 0; --c)
          for (int i = 0; i < here; ++i) {
            if (t[b0 + i] && (rest(i) < 1 || rest(i) > W * tpw[i])) bad = "a last block of no size";
            const bool f = cls(W * tpw[i]) == c, l = cls(rest(i)) == c;
            small += l && !f;
            if (f) from[i] = base;
            base += f ? nb[i] - 1 : 0;
            if (l) last[i] = base++;
          }
        if (base != all) bad = "a class outside the eight";
      }
      std::set<std::pair<int, int>> taken;
      int before = kPagedClasses;
      for (int place = 0; place < all; ++place) {
        int who = -1;
        for (int i = 0; i < here; ++i)
          if ((from[i] <= place && place < from[i] + nb[i] - 1) || place == last[i]) {
            if (who >= 0) bad = "two blocks at one place";
            who = i;
          }
        if (who < 0) { bad = "no block at a place"; continue; }
        const int blk = place == last[who] ? nb[who] - 1 : place - from[who];
        if (blk < 0 || blk >= nb[who] || !taken.insert({who, blk}).second) bad = "a block twice, or none of the sequence's";
        const int c = cls(blk == nb[who] - 1 ? rest(who) : W * tpw[who]);
        if (sort && c > before) bad = "a larger block behind a smaller one's class";
        before = c;
      }
      if ((int)taken.size() != all) bad = "a block without a place";
    }
    std::printf("%d %d %s.\n", sorted, small, bad);
  }
}
"""


def test_every_block_has_a_place(tmp_path):
    src, exe = tmp_path / "deal.cc", tmp_path / "deal"
    src.write_text(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + libbuild.CSRC, str(src), "-o", str(exe)],
                   check=True)
    rng = random.Random(3)
    lines = []
    for _ in range(3000):
        Hkv = rng.choice([1, 2, 4, 8, 16])
        n = int(round(200000 ** rng.random()))
        B = rng.choice([1, 2, 7, 48, 63, 64, 65, 130])
        lens = [rng.choice([0, 1, n, rng.randint(0, n), int(round(n ** rng.random()))]) for _ in range(B)]
        dense = rng.randrange(2)
        lines.append("%d %d %d %d %d %d %d %d %s" % (B, Hkv * rng.choice([1, 4, 17]), Hkv, rng.choice([64, 128]),
                                                     rng.randrange(2), n, 32 * rng.choice([1, 2, 4, 8, 16]), dense,
                                                     " ".join(map(str, lens))))
    out = subprocess.run([str(exe)], input="\n".join(lines), text=True, capture_output=True, check=True).stdout
    out = [x.split(" ", 2) for x in out.strip().split("\n")]
    assert len(out) == len(lines)
    wrong = [(a, o) for a, o in zip(lines, out) if o[2] != "."]
    assert not wrong, wrong[:3]
    assert sum(int(o[0]) > 0 for o in out) > 1000 and sum(int(o[1]) for o in out) > 1000
