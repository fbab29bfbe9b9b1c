"""Rows that share memory (CPU): the host's answer (csrc/mala_rows.h, compiled here) against a look at
every pair of rows, and the calls that have to refuse such outputs."""
import ctypes
import itertools
import random
import shutil
import subprocess

import pytest
import torch

import paper_2609_32712_amd as mala
from paper_2609_32712_amd import build as libbuild
from test_rope_block_abi import BAD, _block_cache, _refused, _rope, _rows, _turn

CXX = shutil.which("g++")
needs_cxx = pytest.mark.skipif(CXX is None, reason="needs g++")

PROGRAM = r"""
#include <cstdio>
#include "mala_rows.h"
using namespace mala;
static bool get(Rows& r) {
  long b, w, s[3], n[3];
  if (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld", &b, &w, s, s + 1, s + 2, n, n + 1, n + 2) != 8) return false;
  r = {(uintptr_t)b, w, {s[0], s[1], s[2]}, {n[0], n[1], n[2]}};
  return true;
}
int main(int argc, char**) {
  Rows r, s;
  if (argc > 1)
    while (get(r) && get(s)) std::printf("%d\n", (int)rows_meet(r, s));
  else
    while (get(r)) std::printf("%d\n", (int)rows_overlap(r));
}
"""


def _ask(tmp_path, lines, *args):
    src, exe = tmp_path / "rows.cc", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I" + libbuild.CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe), *args], input="\n".join(" ".join(map(str, x)) for x in lines), text=True,
                         capture_output=True, check=True).stdout.split()
    assert len(out) == len(lines)
    return [int(x) for x in out]


def _places(r):
    base, _, s, n = r[0], r[1], r[2:5], r[5:8]
    return [base + sum(i * a for i, a in zip(at, s)) for at in itertools.product(*map(range, n))]


def _random(rng):
    w = 16 * rng.choice([1, 2, 8])
    nested = rng.random() < 0.4
    n = [rng.randint(1, 6) for _ in range(3)]
    s = [16 * rng.randint(0, 30) for _ in range(3)]
    if nested:
        step = w
        for i in rng.sample(range(3), 3):
            s[i] = step + 16 * rng.choice([0, 0, 1, 5]) * rng.randint(0, 1)
            step = s[i] * n[i]
    return [16 * rng.randint(0, 60), w] + s + n


@needs_cxx
def test_own_rows(tmp_path):
    rng = random.Random(1)
    rows = [_random(rng) for _ in range(4000)]
    want = []
    for r in rows:
        at = sorted(_places(r))
        want.append(int(any(b - a < r[1] for a, b in zip(at, at[1:]))))
    assert 800 < sum(want) < 3200
    assert _ask(tmp_path, rows) == want
    # large ones: rows side by side in every order, 16 bytes short of it, and strides that do not nest
    cases = [([0, 256, 256 * 40, 256, 256 * 40 * 70000, 70000, 40, 100], 0),
             ([0, 256, 256 * 70000, 256, 256 * 40 * 70000, 40, 70000, 100], 0),
             ([0, 256, 256 * 40 - 16, 256, 256 * 40 * 70000, 70000, 40, 100], 1),
             ([0, 256, 256, 256, 1 << 40, 2, 2, 1], 1), ([0, 256, 256, 256, 1 << 40, 1, 2, 1], 0),
             ([0, 256, 3 * 256, 2 * 256, 1 << 40, 2, 2, 2], 0), ([0, 256, 3 * 256, 2 * 256, 1 << 40, 3, 4, 2], 1),
             ([0, 256, 0, 256, 1024, 1, 4, 1], 0), ([0, 256, 0, 256, 1024, 2, 4, 1], 1),
             ([0, 256, 1 << 59, 1 << 58, 1 << 50, 2, 2, 2], 0),
             # (strides no memory has, and more steps than are taken: not told, and refused)
             ([0, 256, 1 << 60, 3 << 59, 1 << 58, 2, 2, 4], 2),
             ([0, 32, 16 * 100003, 16 * 99991, 1 << 45, 90000, 90000, 1], 2)]
    assert _ask(tmp_path, [c for c, _ in cases]) == [x for _, x in cases]


@needs_cxx
def test_rows_of_two_tensors(tmp_path):
    rng = random.Random(2)
    pairs, want = [], []
    for _ in range(4000):
        x, y = _random(rng), _random(rng)
        if rng.random() < 0.3:           # slices of one tensor: the same strides
            y[2:5] = x[2:5]
        pairs.append(x + y)
        want.append(int(any(-x[1] < a - b < y[1] for a, b in itertools.product(_places(x), _places(y)))))
    assert 800 < sum(want) < 3600
    assert _ask(tmp_path, pairs, "two") == want
    # queries, keys and values of one projection of 32 + 8 + 8 heads, and 16 bytes too far
    row = 48 * 256
    q = [1 << 20, 256, 0, 256, row, 1, 32, 1 << 20]
    k = [(1 << 20) + 32 * 256, 256, 0, 256, row, 1, 8, 1 << 20]
    far = [k[0] - 16] + k[1:]
    batches = [q[:2] + [row << 10] + q[3:5] + [9, 32, 1 << 10], k[:2] + [row << 10] + k[3:5] + [9, 8, 1 << 10]]
    assert _ask(tmp_path, [q + k, k + q, q + far, far + q, batches[0] + batches[1]], "two") == [0, 0, 1, 1, 0]


@needs_cxx
def test_large_tensors_and_their_slices_are_told_apart(tmp_path):
    # axes of any size in any order, padded or not; two slices of the heads, and of every other head
    rng = random.Random(3)
    own, pairs, want = [], [], []
    for _ in range(3000):
        w = rng.choice([128, 256, 512])
        heads = rng.randint(2, 300)
        n = {"b": int(2 ** rng.uniform(0, 12)), "h": heads, "t": int(2 ** rng.uniform(0, 21))}
        step, stride = w, {}
        for axis in rng.sample("bht", 3):
            stride[axis] = step + 16 * rng.choice([0, 0, 0, 1, 7, 64])
            step = stride[axis] * n[axis]
        rows = lambda first, count, every=1: [(1 << 20) + first * stride["h"], w, stride["b"], every * stride["h"],
                                              stride["t"], n["b"], count, n["t"]]
        own.append(rows(0, heads))
        cut = rng.randint(1, heads - 1)
        pairs.append(rows(0, cut) + rows(cut, heads - cut))
        want.append(0)
        pairs.append(rows(0, -(-heads // 2), 2) + rows(1, heads // 2, 2))
        want.append(0)
        pairs.append(rows(0, cut + 1) + rows(cut, heads - cut))
        want.append(1)
    assert not any(_ask(tmp_path, own))
    assert _ask(tmp_path, pairs, "two") == want


def test_outputs_that_share_rows_are_refused():
    # (rows of 256 bytes, 2 x 4 x 4 of them, 8 KB to a batch; in is 1 << 20, out 1 << 30)
    at = 1 << 21
    for q, k in ((dict(), dict(x=at)),                                     # one output for both
                 (dict(), dict(x=at, out=(1 << 30) + 240)),
                 (dict(ot=2048, ob=8192), dict(x=at, out=(1 << 30) + 768, ot=2048, ob=8192, oh=256)),
                 (dict(), dict(x=1 << 30, out=at)),                        # keys read where queries are written
                 (dict(x=at), dict(x=1 << 22, out=at)),                    # and the other way round
                 (dict(out=1 << 20), dict(x=1 << 20, out=at))):            # queries turned in place are the keys
        _refused(_rope(q=_rows(**q), k=_rows(**k)), BAD)
        assert b"shares memory with" in mala.load_library().mala_last_error()


@pytest.mark.parametrize("kw", [dict(oh=128, ot=128), dict(ob=1024, ot=1024), dict(oh=128, ot=256, ob=2048),
                                dict(oh=128, ot=504, ob=4096), dict(ob=128, oh=1024, ot=192)])
def test_rows_of_an_output_that_overlap_are_refused(kw):
    # (two, four tokens of four heads of 128 elements)
    _refused(_rope(q=_rows(**kw)), BAD)
    _refused(_rope(k=_rows(**kw)), BAD)
    assert b"rows of the output of k overlap" in mala.load_library().mala_last_error()


def test_queries_into_new_rows_are_refused():
    # (queries of 4 heads, 8 tokens of 1024 elements; new rows of 4 heads 1024 elements apart too)
    for dtype in (mala.CACHE_BF16, mala.CACHE_E4M3, mala.CACHE_E4M3_BLOCK):
        cache = ctypes.byref(_block_cache(dtype=dtype, page_stride=8 * 32 * 128, v_block_scale=1 << 40,
                                          k_block_scale=1 << 41))
        lib = mala.load_library()
        for k, v, x, out in ((1 << 30, 1 << 32, 1 << 20, 1 << 30), (1 << 32, 1 << 30, 1 << 20, 1 << 30),
                             (1 << 32, (1 << 30) + 7 * 2048 + 768, 1 << 20, 1 << 30),
                             (1 << 30, 1 << 32, (1 << 30) - 256, (1 << 30) - 256)):
            _refused(lib.mala_paged_rope_write(_rows(x=x, out=out), k, v, 1024, 128, 16, _turn(), cache, 8, None),
                     BAD)
            assert b"the output of q shares memory with" in lib.mala_last_error()


def test_block_scales_among_the_pages_are_refused():
    # (10 pages of 4 heads of 32 rows of 128 bytes, 160 KB of K and of V; 80 bytes of scales each)
    lib, k, v, far = mala.load_library(), 1 << 30, 1 << 32, 1 << 40
    rows = dict(k_pages=k, v_pages=v, page_stride=4 * 32 * 128)
    wide = dict(k_pages=k, v_pages=k + 128, token_stride=256, head_stride=32 * 256, page_stride=4 * 32 * 256 + 64)
    for pages, bad in ((rows, (k, v, k + 77, v + 10 * 16384 - 1, k - 79)), (wide, (k, k + 4 * 32 * 256 - 1, k + 200))):
        for at in bad:
            for scales in (dict(k_block_scale=at, v_block_scale=far), dict(k_block_scale=far, v_block_scale=at)):
                c = ctypes.byref(_block_cache(**pages, **scales))
                _refused(lib.mala_paged_write(1 << 20, 1 << 22, 512, 128, 16, c, 4, None), BAD)
                assert b"block scales share memory with the pages" in lib.mala_last_error()
                _refused(lib.mala_paged_rope_write(None, 1 << 20, 1 << 22, 512, 128, 16, _turn(), c, 4, None), BAD)


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 32])
def test_block_scales_between_and_behind_pages_are_taken(P):
    # pages and scales in one allocation: the scales behind the last page, and in a gap behind each
    # head's rows that nothing else uses
    import block_util as bu
    N, Hkv, D, T = 6, 2, 64, 40
    n = N * Hkv * (P // 16)
    x = torch.randn((2, Hkv, T, D), device="cuda").bfloat16()
    slots = torch.arange(T, dtype=torch.int32, device="cuda")
    want = bu.block_cache(mala, N, Hkv, P, D)
    mala.mala_paged_write(x[0], x[1], slots, want[0])
    for gap in (0, 64):                  # (bytes behind a head's rows)
        head = P * D + gap
        one = torch.zeros(2 * N * Hkv * head + 2 * n, dtype=torch.uint8, device="cuda")
        k, v = (one[i * N * Hkv * head:(i + 1) * N * Hkv * head].view(N, Hkv, head)[..., :P * D]
                .view(N, Hkv, P, D).view(torch.float8_e4m3fn) for i in range(2))
        at = [2 * N * Hkv * head, 2 * N * Hkv * head + n] if not gap else [P * D, head + P * D]
        ks, vs = (one[a:a + n].view(N, Hkv, P // 16).view(torch.float8_e8m0fnu) for a in at)
        mala.mala_paged_write(x[0], x[1], slots, mala.PagedCache(k, v, ks, vs))
        for a, b in zip((k, v, ks, vs), want[1:]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        if gap:
            bad = one[P * D - 1:P * D - 1 + n].view(N, Hkv, P // 16).view(torch.float8_e8m0fnu)
            with pytest.raises(mala.MalaError, match="share memory with the pages"):
                mala.mala_paged_write(x[0], x[1], slots, mala.PagedCache(k, v, vs, bad))


@pytest.mark.gpu
def test_outputs_side_by_side_are_taken():
    # queries and keys into slices of one tensor, of heads in turns, and of batches inside tokens
    f, _ = mala.rope_frequencies(128, device="cuda")
    q, k = (torch.randn((3, h, 50, 128), device="cuda").bfloat16() for h in (4, 2))
    want = mala.rope(q, k, None, f)
    one = torch.zeros((50, 3, 9, 128), dtype=torch.bfloat16, device="cuda")
    heads = one.permute(1, 2, 0, 3)
    for qo, ko in ((heads[:, :4], heads[:, 4:6]), (heads[:, :8:2], heads[:, 1:4:2]), (heads[:, 5:], heads[:, 1:3])):
        one.zero_()
        mala.mala_rope(q, k, qo, ko, None, f)
        assert torch.equal(qo, want["q"]) and torch.equal(ko, want["k"])
        assert int((one != 0).any(-1).sum()) == 50 * 3 * 6
    for qo, ko in ((heads[:, :4], heads[:, 3:5]), (heads[:, :4], heads[:, 0:4:2])):
        with pytest.raises(mala.MalaError):
            mala.mala_rope(q, k, qo, ko, None, f)
