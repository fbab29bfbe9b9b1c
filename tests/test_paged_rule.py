"""The paged decode's decision and its early form (csrc/mala_paged_dispatch.h), on the CPU."""
import shutil
import subprocess

import pytest

from paper_2609_32712_amd import build as libbuild

CXX = shutil.which("g++")
pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")

PROGRAM = r"""
#include <cmath>
#include <cstdio>
#include "mala_paged_dispatch.h"
using namespace mala;
// V of a tile is fetched by the early test, with a log-sum that can be a step of fp32 above the one
// that decides: whatever the size of the scores, a tile that is retained has to be fetched.
int main() {
  long wrong = 0, all = 0, spared = 0;
  for (int e = -10; e < 60; ++e)
    for (int i = 0; i < 16; ++i)
      for (float sign : {1.f, -1.f})
        for (float thr2 : {-3.f, -15.3f, -40.25f, 0.7f, -170.f})
          for (int steps = 0; steps <= 1; ++steps) {
            const float before = sign * std::ldexp(1.f + i / 16.f, e);
            const float after = steps ? std::nextafter(before, -INFINITY) : before;
            // the smallest maxima that are retained, and some above
            float mt = after + thr2;
            while (paged_retains(mt, after, thr2)) mt = std::nextafter(mt, -INFINITY);
            for (int k = 0; k < 6; ++k, mt = std::nextafter(mt, INFINITY)) {
              if (!paged_retains(mt, after, thr2)) continue;
              ++all;
              wrong += !paged_may_retain(mt, before, thr2);
            }
            // far below the tolerance nothing is fetched
            spared += !paged_may_retain(before + thr2 - 1.f - std::fabs(before) * 1e-6f, before, thr2);
          }
  // no tile is retained against a log-sum of infinity or NaN, whichever comes first
  wrong += paged_retains(1.f, INFINITY, -5.f) || paged_retains(1.f, NAN, -5.f) || paged_may_retain(1.f, NAN, -5.f);
  std::printf("%ld %ld %ld\n", wrong, all, spared);
}
"""


def test_a_retained_tile_is_never_ruled_out_early(tmp_path):
    src, exe = str(tmp_path / "rule.cpp"), str(tmp_path / "rule")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + libbuild.CSRC, src, "-o", exe],
                   check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    wrong, total, spared = map(int, out.split())
    assert wrong == 0 and total > 100000
    assert spared == 70 * 16 * 2 * 5 * 2
