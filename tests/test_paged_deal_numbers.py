"""What the workgroups of a ragged paged decode work on, as the kernel deals them now (CPU): a sequence's
full blocks by their tiles and its last one by what is left.  The blocks of a sequence keep the numbers
under which the join looks for them, its tiles are some wavefront's, once, and the calls of
test_paged_long.py reach the branches they are there for."""
import random
import shutil
import subprocess

import pytest

from paper_2609_32712_amd import build as libbuild

CXX = shutil.which("g++")
pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")

# share_of, place by place, and the runs of a block's wavefronts
PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "mala_paged_dispatch.h"
using namespace mala;
struct Share { int b, blk, blocks, first, tpw; };
static Share share_of(const std::vector<int>& t, unsigned per_block, unsigned unit, int W, bool sorted, int at) {
  int before = 0;
  for (int b0 = 0; b0 < (int)t.size(); b0 += 64) {
    const int here = std::min(64, (int)t.size() - b0);
    std::vector<int> nb(here), end(here), tpw(here), from(here), last(here);
    int all = 0;
    bool sort = false;
    for (int i = 0; i < here; ++i) {
      nb[i] = paged_blocks_of(t[b0 + i], per_block);
      tpw[i] = paged_run_tiles(t[b0 + i], nb[i], unit, W);
      from[i] = all;
      end[i] = all += nb[i];
      last[i] = all - 1;
      sort |= tpw[i] > 4;
    }
    if (at >= before + all) {
      before += all;
      continue;
    }
    if (sorted && sort) {
      int base = 0;
      for (int c = kPagedClasses - 1; c >= 0; --c)
        for (int i = 0; i < here; ++i) {
          if (paged_run_class(W * tpw[i], per_block, 1) == c) {
            from[i] = base;
            base += nb[i] - 1;
          }
          if (paged_run_class(t[b0 + i] - (nb[i] - 1) * W * tpw[i], per_block, 1) == c) last[i] = base++;
        }
    }
    const int place = at - before;
    for (int i = 0; i < here; ++i)
      if ((from[i] <= place && place < from[i] + nb[i] - 1) || place == last[i])
        return {b0 + i, place == last[i] ? nb[i] - 1 : place - from[i], nb[i], before + end[i] - nb[i], tpw[i]};
    return {-2, 0, 0, 0, 0};
  }
  return {-1, 0, 0, 0, 0};
}
int main() {
  int B, Hq, Hkv, D, e4m3, max_len, split, dense;
  while (std::scanf("%d %d %d %d %d %d %d %d", &B, &Hq, &Hkv, &D, &e4m3, &max_len, &split, &dense) == 8) {
    const PagedPlan x = paged_plan(B, Hq, Hkv, D, e4m3, max_len, split, dense);
    const int W = paged_runs(x.mode);
    std::vector<int> t(B);
    unsigned total = 0;
    int longest = 0, runs = 0, cut = 0;
    for (int& n : t) {
      if (std::scanf("%d", &n) != 1) return 1;
      n = (std::min(n, max_len) + kPagedTile - 1) / kPagedTile;
      total += n;
      longest = std::max(longest, n);
    }
    const unsigned per_block = paged_block_tiles(total, longest, B, x.target, x.ragged, x.min_tpw, x.unit, W);
    const bool dealt = B > 1 && (long)x.blocks * Hkv * x.nchunk > kNumCus;
    const char* bad = "";
    std::vector<std::vector<int>> covered(B);
    std::vector<int> number(x.blocks, -1);
    for (int b = 0; b < B; ++b) covered[b].assign(t[b], 0);
    int blocks = 0, of_last = 0, apart = 0;
    for (int at = 0; at < x.blocks; ++at) {
      const Share s = share_of(t, per_block, x.unit, W, dealt, at);
      if (s.b == -1) continue;
      if (s.b < 0) { bad = "no block at a place"; break; }
      ++blocks;
      if (s.blk < 0 || s.blk >= s.blocks || s.first < 0 || s.first + s.blk >= x.blocks) { bad = "a number that is not the sequence's"; break; }
      if (number[s.first + s.blk] >= 0) bad = "one number for two blocks";
      number[s.first + s.blk] = s.b;
      apart += s.first + s.blk != at;
      for (int w = 0; w < W; ++w) {
        const int lo = std::min(t[s.b], (s.blk * W + w) * s.tpw), hi = std::min(t[s.b], lo + s.tpw);
        if (x.unit > 1 && lo % x.unit && lo < hi) bad = "a run that does not start with a split";
        for (int k = lo; k < hi; ++k) ++covered[s.b][k];
      }
      of_last += s.blocks > 1 && s.blk == s.blocks - 1;
      runs = std::max(runs, s.tpw);
      cut = std::max(cut, s.blocks);
    }
    int want = 0;
    for (int b = 0; b < B; ++b) {
      const int nb = paged_blocks_of(t[b], per_block);
      for (int k = 0; k < nb && !*bad; ++k)
        if (want + k >= x.blocks || number[want + k] != b) bad = "numbers that do not follow the sequences";
      want += nb;
      for (int n : covered[b])
        if (n != 1) bad = "a tile left out or worked on twice";
    }
    if (blocks != want) bad = "more blocks than places";
    std::printf("%d %d %d %d %d %d %s.\n", apart, of_last, x.mode, runs, cut, (int)dealt, bad);
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("deal")
    src, exe = str(d / "ask.cc"), str(d / "ask")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I" + libbuild.CSRC, src, "-o", exe], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, list(c[:8]) + list(c[8]))) for c in cases)
        out = subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout
        got = [ln.split(" ", 6) for ln in out.splitlines()]
        assert len(got) == len(cases)
        return [dict(zip(("apart", "last", "mode", "run", "cut", "dealt"), map(int, g[:6])), bad=g[6]) for g in got]
    return run


def test_numbers_and_tiles(ask):
    rng = random.Random(11)
    cases = []
    for _ in range(1500):
        Hkv = rng.choice([1, 2, 8, 16])
        B = int(round(2 ** rng.uniform(0, 7.5)))
        n = int(round(2 ** rng.uniform(5, 15)))
        kind = rng.choice(["any", "log", "few"])
        lens = [rng.randint(0, n) if kind == "any" else int(2 ** rng.uniform(0, n.bit_length() - 1)) if kind == "log"
                else rng.choice([0, 1, 40]) for _ in range(B)]
        lens[rng.randrange(B)] = n
        cases.append((B, Hkv * rng.choice([1, 4, 17]), Hkv, rng.choice([64, 128]), rng.choice([0, 1]), n,
                      32 * rng.choice([1, 2, 4, 8, 16, 64]), rng.choice([0, 1]), lens))
    got = ask(cases)
    for c, g in zip(cases, got):
        assert g["bad"] == ".", (c[:8], g)
    # calls whose order changes the places, and with last blocks of their own among them
    assert sum(g["apart"] > 0 for g in got) > 100
    assert sum(g["apart"] > 0 and g["last"] > 0 for g in got) > 100


def test_long_calls_reach_their_branches(ask):
    from test_paged_long import CALLS
    got = ask([(len(c["lens"]), c["Hq"], c["Hkv"], c["D"], int(c["e4m3"]), max(c["lens"]), c["split"],
                int(c["tau"] == 0), c["lens"]) for c in CALLS.values()])
    for (name, c), g in zip(CALLS.items(), got):
        assert g["bad"] == "." and g["mode"] == c["mode"] and g["dealt"] == c["dealt"], name
        # a wavefront looks up the pages of 32 tiles at a time
        assert g["run"] > 32 if c["long"] else g["run"] > 4, (name, g)
        assert g["cut"] >= c["cut"], (name, g)
