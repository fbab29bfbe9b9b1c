"""Large calls of the rotation and of the block-scaled cache: several heads to a workgroup, loads past
the caches, blocks whose tokens lie on both sides of a window of 64, prompts in the largest chunks,
reads of eight rows.  A test on the CPU holds the sizes to the branches they are there for."""
import shutil
import subprocess

import numpy as np
import pytest
import torch

import block_util as bu
import paged_util as pu
import paper_2609_32712_amd as mala
from paper_2609_32712_amd import build as libbuild

CXX = shutil.which("g++")
I32, BF16, F32 = torch.int32, torch.bfloat16, torch.float32
gpu = pytest.mark.gpu

# B, Hq, Hkv, T, D, R, layout, in, out, x order, out order
TURNS = {
    "rows past the caches, half": (1, 32, 8, 16001, 128, 128, 0, BF16, BF16, "tokens", "heads"),
    "rows past the caches, interleaved": (1, 32, 8, 16001, 128, 128, 1, BF16, BF16, "heads", "tokens"),
    "rows past the caches, fp32": (2, 32, 8, 4100, 128, 128, 0, F32, BF16, "heads", "heads"),
    "rows past the caches, heads first": (2, 33, 7, 8200, 128, 128, 0, BF16, BF16, "tokens", "tokens"),
    "rows past the caches, fp32 both, heads first": (1, 32, 8, 8200, 128, 128, 1, F32, F32, "tokens", "tokens"),
    "half a head, heads first": (1, 32, 8, 16001, 128, 64, 0, BF16, BF16, "tokens", "tokens"),
    "half a head": (1, 32, 8, 16001, 128, 64, 0, BF16, F32, "heads", "heads"),
    "small heads": (1, 16, 4, 20001, 64, 32, 1, BF16, BF16, "tokens", "heads"),
    "small heads, half": (3, 13, 4, 7001, 64, 16, 0, F32, BF16, "heads", "heads"),
    "small heads, heads first": (1, 16, 4, 20001, 64, 64, 0, BF16, BF16, "tokens", "tokens"),
}
# kinds of the cache for each: Hq, Hkv, T, D, R, layout
PROMPTS = [(24, 7, 11003, 64, 64, 0), (24, 7, 11003, 64, 32, 1), (33, 8, 16003, 128, 128, 0),
           (33, 8, 16003, 128, 64, 0)]
SPREAD = [600, 1900, 4500]            # tokens: chunks of 2, 7 and 16
READS = [(8, 128, 16, "hpd", [9000, 0, 1, 7777]), (4, 128, 48, "phd", [17000]), (8, 64, 32, "wide", [3000] * 6)]

PROGRAM = r"""
#include <cstdio>
#include "mala_rope_dispatch.h"
using namespace mala;
int main() {
  int T, heads, Hkv, D, R, size;
  while (std::scanf("%d %d %d %d %d %d", &T, &heads, &Hkv, &D, &R, &size) == 6)
    std::printf("%d %d %d\n", rope_heads_per_group(T, heads, D), (int)rope_loads_once(T, heads, D, R, size),
                block_write_plan(T, Hkv, true).chunk);
}
"""


@pytest.mark.skipif(CXX is None, reason="needs g++")
def test_the_sizes_reach_their_branches(tmp_path):
    src, exe = tmp_path / "ask.cc", tmp_path / "ask"
    src.write_text(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + libbuild.CSRC, str(src), "-o", str(exe)],
                   check=True)

    def ask(cases):
        out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), text=True,
                             capture_output=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.strip().split("\n")]

    def turn(c, T):
        B, Hq, Hkv, _, D, R, _, tin = c[:8]
        return (B * T, Hq + Hkv, Hkv, D, R, 4 if tin == F32 else 2)

    got = ask([turn(c, c[3]) for c in TURNS.values()])
    for (name, c), (per, once, _) in zip(TURNS.items(), got):
        assert per > 1 and once == ("past the caches" in name), (name, per, once)
    # last slices that are short, and slices that hold queries and keys
    assert sum((c[1] + c[2]) % per > 0 for c, (per, _, _) in zip(TURNS.values(), got)) >= 6
    assert sum(c[1] % per > 0 for c, (per, _, _) in zip(TURNS.values(), got)) >= 6
    # the pieces they are compared with: a head to a workgroup
    assert all(x[:2] == (1, 0) for x in ask([turn(c, PIECE) for c in TURNS.values()]))
    for Hq, Hkv, T, D, R, _ in PROMPTS:
        (per, _, chunk), (units, _, _) = ask([(T, Hq, Hkv, D, R, 2), (T, Hkv, Hkv, D, R, 2)])
        assert chunk == 16 and per > 1 and per % 2 and Hq % per != 1
        assert units == (2 if D == 64 else 1)
    assert [c for _, _, c in ask([(T, 1, 2, 64, 64, 2) for T in SPREAD])] == [2, 7, 16]


PIECE = 500


def _rows(rng, B, H, T, D, dtype, order):
    x = torch.from_numpy(rng.standard_normal((B, T, H, D) if order == "tokens" else (B, H, T, D),
                                             dtype=np.float32)).to(dtype).cuda()
    return x.transpose(1, 2) if order == "tokens" else x


@gpu
@pytest.mark.parametrize("name", TURNS)
def test_heads_of_a_workgroup(name):
    # the same bits as in calls of few tokens, a head to a workgroup; those against the definition
    B, Hq, Hkv, T, D, R, layout, tin, tout, xo, oo = TURNS[name]
    rng = np.random.default_rng(T + R)
    f, _ = mala.rope_frequencies(R, device="cuda")
    pos = rng.integers(0, 1 << 20, (B, T))
    p = torch.from_numpy(pos).int().cuda()
    q, k = _rows(rng, B, Hq, T, D, tin, xo), _rows(rng, B, Hkv, T, D, tin, xo)
    place = lambda H: (torch.full((B, T, H, D), 9.0, dtype=tout, device="cuda").transpose(1, 2) if oo == "tokens" else
                       torch.full((B, H, T, D), 9.0, dtype=tout, device="cuda"))
    qo, ko = place(Hq), place(Hkv)
    mala.mala_rope(q, k, qo, ko, p, f, layout, 1.25)
    for x, got in ((q, qo), (k, ko)):
        want = torch.empty((B, x.shape[1], T, D), dtype=tout, device="cuda")
        for a in range(0, T, PIECE):
            mala.mala_rope(x[:, :, a:a + PIECE], None, want[:, :, a:a + PIECE], None,
                           p[:, a:a + PIECE].contiguous(), f, layout, 1.25)
        assert torch.equal(got, want)
        at = np.sort(rng.choice(T, 40, replace=False))
        x64, fn = x[:, :, at].double().cpu().numpy(), f.cpu().numpy()
        exact = bu.turned(x64, pos[:, None, at], fn, layout, 1.25)
        bound = bu.turned_bound(x64, fn, layout, 1.25, tout == BF16, 1 << 20)
        assert (np.abs(got[:, :, at].double().cpu().numpy() - exact) <= bound).all()
    if tin == tout:                     # in place
        qi, ki = q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)
        assert qi.stride() == q.stride()
        mala.mala_rope(qi, ki, qi, ki, p, f, layout, 1.25)
        assert torch.equal(qi, qo) and torch.equal(ki, ko)


def _prompt_slots(rng, T, pages, P):
    """Runs of consecutive slots that start anywhere in a page of their own, padding between some."""
    slots, order, used = np.full(T, -1), rng.permutation(pages), 0
    at = 0
    while at < T:
        n = min(int(rng.integers(1, 900)), T - at)
        first = int(rng.integers(0, P))
        k = (first + n - 1) // P + 1
        if used + k > pages:
            break
        i = first + np.arange(n)
        slots[at:at + n] = order[used + i // P] * P + i % P
        used += k
        at += n + (int(rng.integers(0, 3)) if rng.random() < 0.3 else 0)
    return slots


def _two_caches(kind, N, Hkv, P, D):
    both = []
    for _ in range(2):
        if kind == "block":
            both.append(bu.block_cache(mala, N, Hkv, P, D, fill=0x31))
        else:
            k, v = pu.pool(N, Hkv, P, D, kind == "e4m3")
            s = torch.linspace(0.01, 0.02, Hkv).cuda() if kind == "e4m3" else None
            both.append((mala.PagedCache(k, v, s, s), k, v, None, None))
    return both


def _same_bytes(a, b):
    for x, y in zip(a[1:], b[1:]):
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
@pytest.mark.parametrize("Hq,Hkv,T,D,R,layout", PROMPTS)
@pytest.mark.parametrize("kind", ["block", "e4m3", "bf16"])
def test_rope_write_of_long_prompts(kind, Hq, Hkv, T, D, R, layout):
    rng = np.random.default_rng(T)
    P = 16
    N = T // P + 200
    slots = torch.from_numpy(_prompt_slots(rng, T, N, P)).int().cuda()
    assert int((slots >= 0).sum()) > T - 200
    f, _ = mala.rope_frequencies(R, device="cuda")
    pos = torch.from_numpy(rng.integers(0, 100000, T)).int().cuda()
    proj = _rows(rng, 1, Hq + 2 * Hkv, T, D, BF16, "tokens")[0]
    q, kn, vn = proj[:Hq], proj[Hq:Hq + Hkv], proj[Hq + Hkv:]
    turned = [torch.empty((h, T, D), dtype=BF16, device="cuda") for h in (Hq, Hkv)]
    for a in range(0, T, PIECE):
        for x, y in zip((q, kn), turned):
            mala.mala_rope(x[:, a:a + PIECE], None, y[:, a:a + PIECE], None, pos[a:a + PIECE].contiguous(), f, layout)
    caches = _two_caches(kind, N, Hkv, P, D)
    mala.mala_paged_write(turned[1], vn.contiguous(), slots, caches[0][0])
    for tokens_first in (True, False):
        got = mala.paged_rope_write(q, kn, vn, pos, slots, caches[1][0], f, layout, tokens_first=tokens_first)["q"]
        assert torch.equal(got.transpose(0, 1) if tokens_first else got, turned[0])
        _same_bytes(caches[0], caches[1])
    # in place, among the slices of one projection
    mala.mala_paged_rope_write(q, q, kn, vn, pos, slots, caches[1][0], f, layout)
    assert torch.equal(q, turned[0])
    _same_bytes(caches[0], caches[1])


def _spread_slots(rng, T, blocks):
    """Slots as they may lie: the tokens of a block anywhere within 64 consecutive ones, in any order,
    with those of others between; some blocks hold the first and the last token of such a window."""
    slots = np.full(T, -1)
    for block in rng.permutation(blocks):
        at = int(rng.integers(0, T))
        free = at + np.flatnonzero(slots[at:at + 64] < 0)
        n = min(len(free), int(rng.integers(1, 17)))
        pick = rng.choice(free, n, replace=False)
        if n > 1:
            pick[:2] = free[0], free[-1]
            pick = np.unique(pick)
        slots[pick] = 16 * block + rng.permutation(16)[:len(pick)]
    return slots


def test_spread_slots_lie_on_both_sides_of_a_window():
    # blocks whose first token is not a chunk's first one, and whose last one is 64 or more behind the
    # chunk's start: the kernel finds them in its second window
    for T in SPREAD:
        slots, chunk = _spread_slots(np.random.default_rng(T), T, T // 4), min(16, T // 256)
        late = 0
        for block in np.unique(slots[slots >= 0] // 16):
            at = np.flatnonzero((slots >= 0) & (slots // 16 == block))
            assert at[-1] - at[0] < 64
            late += at[-1] - at[0] // chunk * chunk >= 64
        assert late >= 10, (T, late)


@gpu
@pytest.mark.parametrize("T", SPREAD)
@pytest.mark.parametrize("D,P", [(64, 16), (128, 48)])
def test_writes_of_blocks_across_windows(T, D, P):
    from test_paged_block import Cache
    rng = np.random.default_rng(T)
    blocks = T // 4
    c = Cache(T, -(-blocks // (P // 16)), 2, P, D)
    slots = _spread_slots(rng, T, blocks)
    c.write(slots, order="tokens")
    c.write(slots[::-1].copy())
    # rotated: the same bytes as the turned keys' write
    f, _ = mala.rope_frequencies(D, device="cuda")
    pos = torch.from_numpy(rng.integers(0, 100000, T)).int().cuda()
    x = c.rows(T)
    kn, vn = x[0].cuda(), x[1].cuda()
    q = _rows(rng, 1, 3, T, D, BF16, "tokens")[0]
    got = mala.paged_rope_write(q, kn, vn, pos, torch.from_numpy(slots).int().cuda(), c.cache, f, 1)["q"]
    whole = mala.rope(q, kn, pos, f, 1)
    assert torch.equal(got, whole["q"])
    for i, y in enumerate((whole["k"].cpu(), x[1])):
        bu.write_plain(*c.plain[i], y.double().numpy(), slots)
    c.check()


@gpu
@pytest.mark.parametrize("Hkv,D,P,layout,lens", READS)
@pytest.mark.parametrize("kind", ["block", "e4m3"])
def test_reads_of_many_rows(kind, Hkv, D, P, layout, lens):
    rng = np.random.default_rng(Hkv * D)
    table, N = pu.scatter_tables(rng, lens, P)
    _, k, v, ks, vs = bu.block_cache(mala, N, Hkv, P, D, layout)
    for t in (k, v):
        x = rng.integers(0, 256, t.shape, dtype=np.uint8)
        x[(x & 0x7F) == 0x7F] = 0x7E
        pu.raw(t).copy_(torch.from_numpy(x).cuda())
    for s in (ks, vs):
        s.view(torch.uint8).copy_(torch.from_numpy(rng.integers(100, 150, s.shape, dtype=np.uint8)).cuda())
    heads = torch.linspace(0.01, 0.02, Hkv).cuda()
    cache = mala.PagedCache(k, v, ks, vs) if kind == "block" else mala.PagedCache(k, v, heads, heads)
    cu = np.concatenate([[0], np.cumsum(lens)]) + 5
    total = int(cu[-1]) + 7
    assert total >= 16384
    out = [torch.full((Hkv, total, D), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
    mala.mala_paged_read(cache, torch.from_numpy(table).cuda(), torch.from_numpy(cu).int().cuda(), max(lens), *out)
    for t, s, got in ((k, ks, out[0]), (v, vs, out[1])):
        want = torch.full((Hkv, total, D), 7.0, dtype=BF16, device="cuda")
        values = pu.raw(t).contiguous().view(torch.float8_e4m3fn).float()
        if kind == "block":               # (a power of two: exact)
            values *= torch.exp2(s.view(torch.uint8).float() - 127).repeat_interleave(16, 2)[..., None]
        else:                             # (one product in fp32, rounded once)
            values *= heads[None, :, None, None]
        for b, n in enumerate(lens):
            at = torch.arange(n)
            rows = values[torch.from_numpy(table[b]).long()[at // P].cuda(), :, (at % P).cuda()]
            want[:, cu[b]:cu[b] + n] = rows.transpose(0, 1).to(BF16)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
