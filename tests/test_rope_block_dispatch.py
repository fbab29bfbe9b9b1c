"""How rotations and block-scaled writes are shared out (csrc/mala_rope_dispatch.h), on the CPU: a
small C++ program compiled against the header does what the kernels do with it.  Every token and head
has to be some wavefront's, once, and the grids have to fit the limits that the calls check."""
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
#include "mala_rope_dispatch.h"
using namespace mala;
int main() {
  int T, Hkv, heads, D, rope;
  while (std::scanf("%d %d %d %d %d", &T, &Hkv, &heads, &D, &rope) == 5) {
    const char* bad = "";
    const BlockWritePlan x = block_write_plan(T, Hkv, rope);
    const int64_t chunks = ((int64_t)T + x.chunk - 1) / x.chunk;
    const int parts = block_write_parts(Hkv, x.units);
    if (x.chunk < 1 || x.chunk > kBlockChunk || x.units < 1) bad = "sizes";
    if (x.groups != chunks * parts) bad = "groups";
    if (x.groups > std::max<int64_t>(chunks, 16 * kNumCus)) bad = "too many groups";
    // heads of K and V: each some wavefront's, once (the kernel's ranges)
    std::vector<int> seen(2 * Hkv);
    for (int part = 0; part < parts; ++part) {
      const int lo = part * 4 * x.units, hi = std::min(lo + 4 * x.units, 2 * Hkv);
      if (lo >= hi) bad = "a part without heads";
      for (int w = 0; w < 4; ++w)
        for (int u = lo + w; u < hi; u += 4) ++seen[u];
    }
    for (int n : seen)
      if (n != 1) bad = "a head not taken once";
    const int per = rope_heads_per_group(T, heads, D);
    const int64_t slices = (heads + per - 1) / per;
    if (per < 1 || per > heads || slices > 65535) bad = "slices";
    if ((int64_t)rope_tokens(D) * D != 4096) bad = "tokens of a workgroup";
    // 32-bit numbers of the workgroups
    if (((int64_t)T + rope_tokens(D) - 1) / rope_tokens(D) * slices > UINT32_MAX) bad = "workgroups";
    std::printf("%s\n", *bad ? bad : "ok");
  }
}
"""


def test_every_token_and_head_once(tmp_path):
    src, exe = tmp_path / "plan.cc", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + libbuild.CSRC, str(src), "-o", str(exe)],
                   check=True)
    rng = random.Random(1)
    cases = [(1, 1, 1, 64, 0), (1, 1, 1, 128, 1), (2 ** 29 - 32, 8, 40, 128, 1), (2 ** 30 - 64, 1, 2, 64, 0),
             (1, 1000, 65535, 128, 1), (4096, 131, 131070, 64, 0)]
    for _ in range(4000):
        size = lambda most: int(round(most ** rng.random()))
        cases.append((size(1 << 22), size(200), size(400), rng.choice([64, 128]), rng.randrange(2)))
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), text=True,
                         capture_output=True, check=True).stdout.split("\n")
    wrong = [(c, o) for c, o in zip(cases, out) if o != "ok"]
    assert not wrong, wrong[:5]


def _lead(slots, chunk):
    """The kernel's rule in words: {first token of a block: its tokens}, for chunks of the tokens."""
    found = {}
    for t0 in range(0, len(slots), chunk):
        todo = [t for t in range(t0, min(t0 + chunk, len(slots))) if slots[t] >= 0]
        while todo:
            t = todo[0]
            block = slots[t] // 16
            here = [n for n in range(t0, min(t0 + 64, len(slots))) if slots[n] >= 0 and slots[n] // 16 == block]
            todo = [n for n in todo if n not in here]
            before = [n for n in range(max(t - 63, t0 - 64, 0), t0) if slots[n] >= 0 and slots[n] // 16 == block]
            if before:
                continue
            late = range(t0 + 64, min(t0 + 64 + t - t0, len(slots))) if chunk > 1 else ()
            found.setdefault(t, here + [n for n in late if slots[n] >= 0 and slots[n] // 16 == block])
    return found


@pytest.mark.parametrize("chunk", [1, 2, 7, 16])
def test_every_token_follows_one_first_token(chunk):
    # slots as the contract has them: the tokens of a block within 64 consecutive tokens, any order
    rng = random.Random(chunk)
    for _ in range(60):
        n = rng.randint(1, 400)
        slots = [-1] * n
        for block in rng.sample(range(100), rng.randint(1, 40)):
            at = rng.randint(0, n - 1)
            free = [t for t in range(at, min(at + 64, n)) if slots[t] < 0]
            picked = rng.sample(free, min(len(free), rng.randint(1, 16)))
            for t, row in zip(picked, rng.sample(range(16), len(picked))):
                slots[t] = 16 * block + row
        taken = sorted(t for ts in _lead(slots, chunk).values() for t in ts)
        assert taken == [t for t in range(n) if slots[t] >= 0]
