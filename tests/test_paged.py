"""The paged KV cache on the GPU against plain 64-bit forms: page tables, writes, reads, the
decode's attention and its decision rule, and a serving run of them together."""
import math

import numpy as np
import pytest
import torch

import paper_2609_32712_amd as mala
import paged_util as pu

pytestmark = pytest.mark.gpu

I32 = torch.int32


def cuda(a, dtype=I32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


class Batch:
    """Sequences of `lens` in scattered pages, values exact in bf16 and e4m3 (see quarters)."""

    def __init__(self, seed, lens, Hq, Hkv, D, P, e4m3=False, layout="hpd", needle=0.0, ks=None,
                 vs=None, width=None):
        rng = np.random.default_rng(seed)
        self.rng, self.lens, self.Hq, self.Hkv, self.D, self.P = rng, lens, Hq, Hkv, D, P
        self.table, self.N = pu.scatter_tables(rng, lens, P, width=width)
        self.k = [pu.quarters(rng, (Hkv, n, D)) for n in lens]
        self.v = [pu.quarters(rng, (Hkv, n, D)) for n in lens]
        self.q = pu.quarters(rng, (len(lens), Hq, D), 4)
        if needle:      # each head looks for one key: +-1 in the direction of its signs
            for b, n in enumerate(lens):
                for h in range(Hq if n else 0):
                    self.q[b, h] = self.q[b, h] / 4 + needle * torch.sign(
                        self.k[b][h // (Hq // Hkv), rng.integers(n)])
            self.q = torch.round(self.q * 4) / 4
        k, v = pu.pool(self.N, Hkv, P, D, e4m3, layout)
        # every row that is not a valid one holds NaN
        for t in (k, v):
            pu.raw(t).fill_(0x7F) if e4m3 else t.fill_(float("nan"))
        pu.fill(k, self.table, lens, self.k, P)
        pu.fill(v, self.table, lens, self.v, P)
        self.ks = None if ks is None else torch.tensor(ks, dtype=torch.float32)
        self.vs = None if vs is None else torch.tensor(vs, dtype=torch.float32)
        self.cache = mala.PagedCache(k, v, None if ks is None else self.ks.cuda(),
                                     None if vs is None else self.vs.cuda())
        self.scale = float(np.float32(D ** -0.5))

    def seen(self, b):
        n = self.lens[b]
        return (self.table[b, np.arange(n) // self.P] >= 0) & (
            self.table[b, np.arange(n) // self.P] < self.N)

    def plain(self, tau=0.0, split=256):
        out = []
        for b, n in enumerate(self.lens):
            ks = np.ones(self.Hkv) if self.ks is None else self.ks.double().numpy()
            vs = np.ones(self.Hkv) if self.vs is None else self.vs.double().numpy()
            out.append(pu.decode_seq(self.q[b].numpy(), self.k[b].numpy() * ks[:, None, None],
                                     self.v[b].numpy() * vs[:, None, None], self.seen(b),
                                     self.scale, tau, split, n))
        return out

    def decode(self, tau=0.0, split=256, max_len=None, **kw):
        return mala.paged_decode(self.q.to(torch.bfloat16).cuda(), self.cache, cuda(self.table),
                                 cuda(self.lens), max_len or max(max(self.lens), 1), self.scale,
                                 tau, split_tokens=split, **kw)

    def check(self, got, want, out_bf16=False, where=None, clear=None):
        o, lse = got["o"].double().cpu().numpy(), got["lse"].double().cpu().numpy()
        vmax = 2.0 * (1 if self.vs is None else float(self.vs.abs().max()))
        for b, n in enumerate(self.lens):
            if where is not None and b not in where:
                continue
            wo, wl = want[b][0], want[b][1]
            none = np.isneginf(wl)
            assert np.isneginf(lse[b][none]).all() and (o[b][none] == 0).all(), b
            none = none if clear is None else none | ~clear[b]
            if none.all():
                continue
            kmax = 2.0 * (1 if self.ks is None else float(self.ks.abs().max()))
            smax = self.scale * kmax * float(self.q[b].abs().sum(1).max())
            to, tl = pu.decode_bounds(n, smax, vmax, out_bf16)
            assert np.abs(o[b] - wo)[~none].max() <= to, (b, np.abs(o[b] - wo).max(), to)
            assert np.abs(lse[b] - wl)[~none].max() <= tl, (b, np.abs(lse[b] - wl).max(), tl)


LENS = [1, 0, 15, 16, 17, 31, 32, 33, 100, 129, 255, 257, 700]

DENSE = [
    # Hq, Hkv, D, P, e4m3, layout, split
    (4, 2, 128, 16, False, "hpd", 256), (4, 2, 128, 16, True, "hpd", 32),
    (8, 1, 64, 48, False, "phd", 64), (8, 1, 64, 48, True, "phd", 256),
    (5, 5, 128, 32, False, "phd", 96), (7, 1, 64, 16, True, "hpd", 128),
    (40, 2, 128, 64, False, "wide", 256), (33, 1, 64, 256, True, "wide", 512),
    (16, 16, 64, 128, False, "hpd", 4096), (32, 2, 128, 80, True, "phd", 160),
]


@pytest.mark.parametrize("Hq,Hkv,D,P,e4m3,layout,split", DENSE)
def test_decode_dense(Hq, Hkv, D, P, e4m3, layout, split):
    scales = dict(ks=np.linspace(0.5, 1.25, Hkv), vs=np.linspace(1.5, 0.75, Hkv)) if e4m3 else {}
    w = Batch(1, LENS, Hq, Hkv, D, P, e4m3, layout, **scales)
    want = w.plain()
    for out in (torch.float32, torch.bfloat16):
        got = w.decode(split=split, out_dtype=out)
        w.check(got, want, out == torch.bfloat16)
        assert got["head_tiles"].cpu().numpy().tolist() == [x[2].tolist() for x in want]
    # without statistics the same bits
    bare = w.decode(split=split, out_dtype=torch.bfloat16, stats=False)
    assert torch.equal(bare["o"], got["o"]) and torch.equal(bare["lse"], got["lse"])
    c = got["counters"].tolist()
    tiles = sum(int(x[2].sum()) for x in want)
    assert c[mala.CNT_LEGAL] == c[mala.CNT_RETAINED] == tiles and c[mala.CNT_SLOTS] == 32 * tiles


@pytest.mark.parametrize("B,n", [(1, 1), (1, 200), (1, 5000), (3, 2047), (40, 700), (300, 130)])
@pytest.mark.parametrize("D,e4m3", [(128, False), (64, True)])
def test_decode_batches(B, n, D, e4m3):
    rng = np.random.default_rng(B)
    lens = [n] + [int(x) for x in rng.integers(0, n + 1, B - 1)]
    w = Batch(2, lens, 8, 2, D, 16, e4m3)
    w.check(w.decode(split=128), w.plain())


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("tau", [1e-3, 0.1, 1.0, 5.0])
@pytest.mark.parametrize("Hq,Hkv,D,P,e4m3,split", [
    (4, 2, 128, 16, False, 256), (8, 1, 64, 32, True, 64), (20, 1, 128, 48, False, 512),
    (3, 3, 64, 64, False, 32), (8, 2, 128, 16, True, 1024)])
def test_decode_rule(Hq, Hkv, D, P, e4m3, split, tau, many):
    # few splits (up to 512 by the longest cache) are shared by the wavefronts of a workgroup,
    # of many each wavefront takes its own: the same batch several times over the same pages
    w = Batch(3, [1, 0, 33, 64, 500, 1023, 1600], Hq, Hkv, D, P, e4m3, needle=128 / D)
    want = w.plain(tau, split)
    if many:
        copies = 1 + 512 // (7 * Hkv * -(-Hq // Hkv // 16) * -(-1600 // split))
        w.lens, w.table, w.q = w.lens * copies, np.tile(w.table, (copies, 1)), w.q.repeat(copies, 1, 1)
        want = want * copies
    got = w.decode(tau, split)
    # a decision can differ where the test value lies within its rounding of tau: that of the
    # normaliser (a sum of at most 1600 terms) and of the scores
    smax = w.scale * 2 * float(w.q.abs().sum(2).max())
    band = 1700 * pu.U24 + 16 * pu.U24 * (smax + 1)
    clear = [x[4] > band for x in want]
    assert sum(x.sum() for x in clear) >= 0.9 * Hq * len(want)
    w.check(got, want, clear=clear)
    tiles = got["head_tiles"].cpu().numpy()
    for b, x in enumerate(want):
        assert tiles[b][clear[b]].tolist() == x[2][clear[b]].tolist()
    # a bf16 output is another instance of the kernels, with the same decisions; and so without
    # statistics
    for stats in (True, False):
        half = w.decode(tau, split, out_dtype=torch.bfloat16, stats=stats)
        w.check(half, want, True, clear=clear)
        assert torch.equal(half["lse"], got["lse"])
    assert torch.equal(w.decode(tau, split, stats=False)["o"], got["o"])
    c = got["counters"].tolist()
    legal = sum(-(-n // 32) for n in w.lens) * Hq
    assert (c[mala.CNT_LEGAL], c[mala.CNT_RETAINED]) == (legal, int(tiles.sum()))
    kept = sum(int(x[2].sum()) for x in want)
    if all(x.all() for x in clear):
        total = 0
        for b, x in enumerate(want):
            for h in range(Hq):
                total = (total + pu.set_hash(x[3][h], b, h)) & ((1 << 64) - 1)
        assert c[mala.CNT_SET_HASH] & ((1 << 64) - 1) == total
    if tau >= 1.0 and split > 32:
        assert kept < legal


@pytest.mark.parametrize("tau", [0.0, 0.1])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_equals_the_contiguous_decode(D, tau):
    # whole splits: mala_decode with as many splits cuts the cache at the same places
    n, split = 2048, 128
    w = Batch(4, [n, n], 8, 2, D, 32, needle=128 / D)
    got = w.decode(tau, split)
    kc, vc = (torch.stack(x).to(torch.bfloat16).cuda() for x in (w.k, w.v))
    ref = mala.decode(w.q.to(torch.bfloat16).cuda(), kc, vc, w.scale, tau, n // split)
    assert torch.equal(got["head_tiles"], ref["head_tiles"])
    assert got["counters"][mala.CNT_SET_HASH] == ref["counters"][mala.CNT_SET_HASH]
    w.check(got, w.plain(tau, split))


@pytest.mark.parametrize("tau", [0.0, 0.1])
@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_missing_pages_are_masked(e4m3, tau):
    w = Batch(5, [300, 64, 640, 48, 16, 1000], 4, 2, 128, 16, e4m3)
    w.table[0, :9] = -1            # a window: the first pages are gone
    w.table[1, :] = -1             # every page: an empty row
    w.table[2, 1::2] = w.N         # every other page outside the pool: half of every tile
    w.table[3, 2] = np.int32(2 ** 31 - 1)
    w.table[4, 0] = np.int32(-2 ** 31)
    w.table[5, 20:40] = -7         # whole splits of 64
    want = w.plain(tau, 64)
    got = w.decode(tau, 64)
    w.check(got, want)
    assert got["head_tiles"].cpu().numpy().tolist() == [x[2].tolist() for x in want]


@pytest.mark.parametrize("D", [64, 128])
def test_decode_lengths_are_clamped(D):
    w = Batch(6, [100, 64, 200, 32], 4, 2, D, 16)
    want = w.plain()
    q, t = w.q.to(torch.bfloat16).cuda(), cuda(w.table)
    lens = cuda([100, -5, 2 ** 31 - 1, -2 ** 31])
    got = mala.paged_decode(q, w.cache, t, lens, 200, w.scale, 0.0, 64)
    w.check(got, want, where=[0, 2])
    for b in (1, 3):
        assert (got["o"][b] == 0).all() and torch.isneginf(got["lse"][b]).all()


def test_one_page_and_one_head_with_any_stride():
    # the stride of an axis of one entry is never used, whatever it says
    rng = np.random.default_rng(22)
    k, v = (torch.zeros(16 * 64, dtype=torch.bfloat16, device="cuda").as_strided(
        (1, 1, 16, 64), (3, 1, 64, 1)) for _ in range(2))
    cache = mala.PagedCache(k, v)
    new = pu.quarters(rng, (2, 13, 64)).to(torch.bfloat16).cuda()
    new = new.as_strided((2, 1, 13, 64), (13 * 64, 5, 64, 1))
    mala.mala_paged_write(new[0], new[1], cuda(np.arange(13)), cache)
    assert torch.equal(k[0, 0, :13], new[0, 0]) and torch.equal(v[0, 0, :13], new[1, 0])
    q = pu.quarters(rng, (1, 3, 64), 4)
    got = mala.paged_decode(q.to(torch.bfloat16).cuda(), cache, cuda([[0]]), cuda([13]), 16, 0.125, 0.0)
    o, lse, tiles, _, _ = pu.decode_seq(q[0].numpy(), new[0].double().cpu().numpy(),
                                        new[1].double().cpu().numpy(), np.ones(13, bool), 0.125, 0.0,
                                        64, 13)
    to, tl = pu.decode_bounds(13, 0.125 * 2 * float(q.abs().sum(2).max()), 2.0, False)
    assert np.abs(got["o"][0].double().cpu().numpy() - o).max() <= to
    assert np.abs(got["lse"][0].double().cpu().numpy() - lse).max() <= tl
    assert got["head_tiles"].tolist() == [[1, 1, 1]]


def test_decode_shared_pages():
    # two sequences with one prefix: the same pages in both rows
    w = Batch(7, [96, 128], 4, 2, 128, 32)
    w.table[1, :3] = w.table[0, :3]
    w.k[1][:, :96], w.v[1][:, :96] = w.k[0], w.v[0]
    w.check(w.decode(split=32), w.plain())


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_offsets_past_32_bits(e4m3):
    # pages at both ends of pools of more than 2^32 bytes each
    Hq, Hkv, D, P, n = 4, 2, 128, 64, 200
    N = (5 << 30) // (Hkv * P * D * (1 if e4m3 else 2))
    rng = np.random.default_rng(8)
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    k = torch.empty((N, Hkv, P, D), dtype=dtype, device="cuda")
    v = torch.empty((N, Hkv, P, D), dtype=dtype, device="cuda")
    w = Batch(8, [n, n], Hq, Hkv, D, P, e4m3)
    w.table = np.array([[N - 1, 0, N - 2, N // 2], [N - 3, 1, N // 2 + 1, N - 4]], dtype=np.int32)
    w.N = N
    pu.fill(k, w.table, w.lens, w.k, P)
    pu.fill(v, w.table, w.lens, w.v, P)
    w.cache = mala.PagedCache(k, v)
    w.check(w.decode(split=64), w.plain())
    out = mala.paged_read(w.cache, cuda(w.table), cuda([0, n, 2 * n]), n, 2 * n)
    assert torch.equal(out["k"].double().cpu(), torch.cat(w.k, 1))
    assert torch.equal(out["v"].double().cpu(), torch.cat(w.v, 1))
    slots = [(N - 5) * P + 3, (N // 2 + 2) * P]
    new = pu.quarters(rng, (2, Hkv, 2, D)).to(torch.bfloat16)
    mala.mala_paged_write(new[0].cuda(), new[1].cuda(), cuda(slots), w.cache)
    for i, s in enumerate(slots):
        for t, x in ((k, new[0]), (v, new[1])):
            assert torch.equal(pu.raw(t)[s // P, :, s % P].view(dtype).float().cpu(), x[:, i].float())


def test_decode_nan_and_inf():
    w = Batch(9, [100, 100, 100], 4, 2, 128, 16)
    clean = w.decode(split=32)
    q = w.q.clone()
    q[0, 1, 5] = float("nan")
    k = w.cache.k_pages
    page, row = int(w.table[1, 2]), 3
    w.cache.v_pages[int(w.table[2, 0]), 1, 4, 7] = float("inf")
    k[page, 0, row, 0] = float("nan")
    got = mala.paged_decode(q.to(torch.bfloat16).cuda(), w.cache, cuda(w.table), cuda(w.lens), 100,
                            w.scale, 0.0, 32)
    o, lse = got["o"], got["lse"]
    assert o[0, 1].isnan().all() and lse[0, 1].isnan()
    assert o[1, :2].isnan().all() and lse[1, :2].isnan().all()
    assert not o[2, 2:, 7].isfinite().any()
    same = torch.ones_like(o, dtype=torch.bool)
    same[0, 1], same[1, :2], same[2, 2:, 7] = False, False, False
    assert torch.equal(o[same], clean["o"][same])
    for b, h in ((0, 0), (0, 2), (0, 3), (1, 2), (1, 3), (2, 0), (2, 3)):
        assert torch.equal(lse[b, h], clean["lse"][b, h])


def test_decode_scores_of_minus_infinity():
    # keys that hold -inf where the query is positive score -inf: they add nothing, and a
    # sequence that has no other key has no output
    w = Batch(10, [70, 40], 2, 1, 64, 16)
    w.q[:, :, 0] = 1.0
    k = w.cache.k_pages
    for b, rows in ((0, range(30, 70)), (1, range(40))):
        for i in rows:
            k[int(w.table[b, i // 16]), :, i % 16, 0] = -math.inf
            w.k[b][:, i, 0] = -math.inf
    want = w.plain()
    got = w.decode(split=32)
    w.check(got, want)


@pytest.mark.parametrize("Hq,Hkv,D,e4m3,n,tau", [
    (2, 1, 64, True, 140001, 0.0), (3, 1, 128, False, 40000, 0.0), (2, 1, 64, False, 70000, 1e-3),
    (17, 1, 128, True, 9000, 1e-3)])
def test_decode_many_blocks(Hq, Hkv, D, e4m3, n, tau):
    # one long cache and few heads: as many blocks as the launch ever makes, and their join
    w = Batch(12, [n, 3, 0], Hq, Hkv, D, 64, e4m3, needle=128 / D)
    want = w.plain(tau, 256)
    clear = [x[4] > (n + 100) * pu.U24 + 16 * pu.U24 * 30 for x in want]
    assert sum(x.sum() for x in clear) >= 0.5 * Hq * 3
    got = w.decode(tau, 256)
    w.check(got, want, clear=clear)
    tiles = got["head_tiles"].cpu().numpy()
    for b, x in enumerate(want):
        assert tiles[b][clear[b]].tolist() == x[2][clear[b]].tolist()


@pytest.mark.parametrize("Hq,Hkv,D,tau", [(40, 1, 128, 0.0), (66, 2, 64, 0.0), (40, 1, 64, 0.1)])
def test_decode_many_chunks(Hq, Hkv, D, tau):
    # three chunks of heads per KV head, more workgroups than CUs, a number that no round divides
    rng = np.random.default_rng(16)
    w = Batch(16, [0, 1] + rng.integers(1, 150, 99).tolist(), Hq, Hkv, D, 16, needle=128 / D)
    want = w.plain(tau, 64)
    smax = w.scale * 2 * float(w.q.abs().sum(2).max())     # (as for the rule's other batches)
    clear = [x[4] > 250 * pu.U24 + 16 * pu.U24 * (smax + 1) for x in want]
    assert sum(x.sum() for x in clear) >= 0.9 * Hq * len(want)
    got = w.decode(tau, 64)
    w.check(got, want, clear=clear)
    tiles = got["head_tiles"].cpu().numpy()
    for b, x in enumerate(want):
        assert tiles[b][clear[b]].tolist() == x[2][clear[b]].tolist()


@pytest.mark.parametrize("ks,vs", [([-0.5, 1.0], [0.75, -1.25]), ([0.0, 0.25], [0.0, 1.0])])
@pytest.mark.parametrize("tau", [0.0, 0.1])
def test_decode_scales_of_any_sign(ks, vs, tau):
    w = Batch(13, [70, 300], 4, 2, 128, 16, True, ks=ks, vs=vs)
    w.check(w.decode(tau, 64), w.plain(tau, 64))


def test_decode_workspace_contents_do_not_matter():
    # 0xFF bytes are NaN partials and negative block numbers
    w = Batch(14, [3000, 100, 0, 2047], 8, 2, 128, 16, needle=1.0)
    for tau in (0.0, 0.1):
        n = mala.mala_paged_decode_workspace_size(4, 8, 2, 128, 3000, 128)
        assert n > 0
        want = w.decode(tau, 128)
        for fill in (0xFF, 0x7F, 0):
            ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
            got = w.decode(tau, 128, workspace=ws)
            assert torch.equal(got["o"], want["o"]) and torch.equal(got["lse"], want["lse"])
            assert torch.equal(got["head_tiles"], want["head_tiles"])


def test_decode_graphs_that_share_a_workspace():
    # two graphs over different caches and one workspace, replayed in turn with lengths that
    # change between replays (so do the blocks of a sequence) and eager calls in between
    ws = [Batch(15 + i, [3000, 500], 8, 2, 128, 16, needle=1.0) for i in range(2)]
    need = mala.mala_paged_decode_workspace_size(2, 8, 2, 128, 3000, 128)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    runs = []
    for i, w in enumerate(ws):
        r = dict(q=w.q.to(torch.bfloat16).cuda(), t=cuda(w.table), n=cuda([1, 1]), tau=0.1 * i,
                 o=torch.empty((2, 8, 128), device="cuda"), lse=torch.empty((2, 8), device="cuda"))
        call = lambda r=r, w=w, out=None: mala.mala_paged_decode(
            r["q"], w.cache, r["t"], r["n"], 3000, *(out or (r["o"], r["lse"])), None, None, 128,
            work, w.scale, r["tau"])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        r["g"], r["call"] = torch.cuda.CUDAGraph(), call
        with torch.cuda.graph(r["g"]):
            call()
        runs.append(r)
    for lens in ([3000, 500], [64, 500], [1500, 0], [2999, 33], [0, 1], [3000, 500]):
        for r in runs:
            r["n"].copy_(cuda(lens))
            out = torch.empty_like(r["o"]), torch.empty_like(r["lse"])
            r["call"](out=out)
            r["eager"] = out
        for r in runs:
            r["g"].replay()
        torch.cuda.synchronize()
        for r in runs:
            assert torch.equal(r["o"], r["eager"][0]) and torch.equal(r["lse"], r["eager"][1])


def test_decode_does_not_depend_on_the_batch():
    lens = [700, 33, 512, 1]
    w = Batch(11, lens, 8, 2, 128, 16, needle=1.0)
    for tau in (0.0, 0.1):
        whole = w.decode(tau, 128)
        q, t = w.q.to(torch.bfloat16).cuda(), cuda(w.table)
        for b, n in enumerate(lens):
            one = mala.paged_decode(q[b:b + 1], w.cache, t[b:b + 1], cuda([n]), 700, w.scale, tau,
                                    128)
            assert torch.equal(one["head_tiles"][0], whole["head_tiles"][b])
            to, tl = pu.decode_bounds(700, 60.0, 2.0, False)
            assert (one["o"][0] - whole["o"][b]).abs().max() <= 2 * to
            assert (one["lse"][0] - whole["lse"][b]).abs().max() <= 2 * tl
        again = w.decode(tau, 128)
        assert torch.equal(again["o"], whole["o"]) and torch.equal(again["lse"], whole["lse"])


# ------------------------------------------------------------------ page tables
def _update(lens, new, table, ring, state, P, N, T):
    args = [cuda(x) for x in (lens, new, table, ring, state)]
    out = mala.paged_update(*args, T, P, N)
    return args[2], args[3], out


def _same_update(lens, new, table, ring, state, P, N, T):
    """One step on the GPU against the loops; the tables, ring and outputs after it."""
    gt, gr, got = _update(lens, new, table, ring, state, P, N, T)
    table, ring = table.copy(), ring.copy()
    lens_out, cu, slots, pos, out = pu.update_plain(lens, new, table, ring, state, P, N, T)
    for name, a, b in (("table", gt, table), ("ring", gr, ring), ("lens", got["lens"], lens_out),
                       ("cu", got["cu_seqlens"], cu), ("slots", got["slots"], slots),
                       ("positions", got["positions"], pos), ("state", got["free_state"], out)):
        np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=name)
    return lens_out, table, ring, out[:2]


@pytest.mark.parametrize("R,W,P,N,grow", [
    (1, 1, 16, 1, 16), (5, 8, 16, 20, 40), (64, 40, 16, 900, 60), (300, 12, 48, 1500, 200),
    (1024, 4, 16, 2000, 30), (1025, 4, 16, 2500, 30), (2500, 6, 32, 4000, 50), (3, 400, 256, 700, 90000)])
def test_update_steps_match_the_loops(R, W, P, N, grow):
    rng = np.random.default_rng(R)
    table, lens = np.full((R, W), -1, np.int32), np.zeros(R, np.int32)
    C = N + int(rng.integers(0, 5))
    ring = np.concatenate([rng.permutation(N), np.full(C - N, -1)]).astype(np.int32)
    head = int(rng.integers(C))
    ring, state = np.roll(ring, head), np.array([head, N], np.int32)
    refused = 0
    for step in range(5):
        kind = rng.random(R)
        new = lens + np.where(kind < 0.4, 1, np.where(kind < 0.7, rng.integers(0, grow + 1, R), 0))
        new = np.where(kind > 0.85, rng.integers(0, lens + 1), new)
        new = np.minimum(new, W * P).astype(np.int32)
        total = int(np.maximum(new - lens, 0).sum())
        T = [total, total + 100, max(0, total - 7), total // 2, total + 5000][step]
        lens, table, ring, state = _same_update(lens, new, table, ring, state, P, N, T)
        refused += int(state[1] == 0)


def test_update_refuses_in_order_and_keeps_those_that_need_nothing():
    P, W, N = 16, 4, 6
    table = np.full((5, W), -1, np.int32)
    table[3, 0] = 5
    ring = np.array([0, 1, 2, 3, 4, -1], np.int32)
    lens = np.array([0, 0, 0, 3, 0], np.int32)
    new = np.array([20, 64, 1, 9, 0], np.int32)     # 2, 4, 1, 0 and 0 pages; 5 are free
    out = _same_update(lens, new, table, ring, np.array([0, 5], np.int32), P, N, 200)
    assert out[0].tolist() == [20, 0, 0, 9, 0]


def test_update_odd_inputs():
    # lengths outside the table's rows, a state outside the ring, page numbers outside the
    # pool, no tokens at all, more pages given back than the ring has room for
    rng = np.random.default_rng(3)
    table = rng.integers(-3, 12, (6, 4)).astype(np.int32)
    ring = rng.integers(-3, 12, 10).astype(np.int32)
    lens = np.array([5, -7, 64, 2 ** 31 - 1, 40, 0], np.int32)
    new = np.array([6, 20, 0, -2 ** 31, 2 ** 31 - 1, 0], np.int32)
    for state in ([3, 4], [-5, 4], [99, 4], [9, 99], [2, -1]):
        _same_update(lens, new, table, ring, np.array(state, np.int32), 16, 10, 150)
    _same_update(lens, lens, table, ring, np.array([1, 3], np.int32), 16, 10, 0)


def test_update_without_positions():
    P, N = 16, 8
    ring, state = cuda(np.arange(N)), cuda([0, N])
    z = lambda n: torch.full((n,), -9, dtype=I32, device="cuda")
    table, slots = torch.full((2, 4), -1, dtype=I32, device="cuda"), z(40)
    mala.mala_paged_update(cuda([0, 0]), cuda([3, 17]), table, ring, state, z(2), z(3), slots, None,
                           z(4), P, N)
    want = list(range(3)) + [16 + i for i in range(16)] + [32] + [-1] * 20
    assert slots.tolist() == want


# ------------------------------------------------------------------ writes and reads
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hkv,D,P,layout,source,T", [
    (1, 64, 16, "hpd", "heads", 1), (2, 128, 16, "hpd", "tokens", 37), (5, 64, 48, "phd", "tokens", 300),
    (8, 128, 32, "wide", "heads", 1000), (3, 128, 64, "phd", "heads", 129)])
def test_write(Hkv, D, P, layout, source, T, e4m3):
    rng = np.random.default_rng(T)
    N = pu.pages_of(T, P) + 3
    k, v = pu.pool(N, Hkv, P, D, e4m3, layout)
    old = rng.integers(0, 120, (2, N, Hkv, P, D)).astype(np.uint8)
    for i, t in enumerate((k, v)):
        x = torch.from_numpy(old[i])
        pu.raw(t).copy_(x.cuda() if e4m3 else x.to(torch.bfloat16).cuda())
    before = [pu.raw(t).cpu().clone() for t in (k, v)]
    x = torch.from_numpy(rng.standard_normal((2, Hkv, T, D)) * 40).to(torch.bfloat16)
    x[0, 0, 0, :6] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1e30, -0.0, 1e-30])
    if source == "tokens":        # slices of one [T, 2, Hkv, D] projection
        both = x.permute(2, 0, 1, 3).contiguous().cuda()
        kn, vn = both[:, 0].transpose(0, 1), both[:, 1].transpose(0, 1)
    else:
        kn, vn = x[0].cuda(), x[1].cuda()
    slots = rng.permutation(N * P)[:T].astype(np.int64)
    slots[rng.random(T) < 0.2] = -1
    if T > 5:
        slots[3], slots[4] = N * P, 2 ** 31 - 1
    ks = torch.linspace(0.05, 0.3, Hkv) if e4m3 else None
    vs = torch.linspace(0.4, 0.1, Hkv) if e4m3 else None
    cache = mala.PagedCache(k, v, ks.cuda() if e4m3 else None, vs.cuda() if e4m3 else None)
    mala.mala_paged_write(kn, vn, cuda(slots), cache)
    for i, (t, s) in enumerate(((k, ks), (v, vs))):
        want = before[i]
        for j in range(T):
            if 0 <= slots[j] < N * P:
                row = x[i, :, j]
                row = pu.e4m3_of(row, s[:, None]).view(torch.uint8) if e4m3 else row
                want[slots[j] // P, :, slots[j] % P] = row
        got = pu.raw(t).cpu()
        if not e4m3:
            want, got = want.view(torch.int16), got.view(torch.int16)
        assert torch.equal(got, want)


@pytest.mark.parametrize("scale", [1.0, 0.0123, 3.7])
def test_e4m3_rounding_of_every_bf16(scale):
    # all 65536 bf16 values, through the write, and every e4m3 byte back through the read
    x = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).view(1, 512, 128)
    k, v = pu.pool(32, 1, 16, 128, e4m3=True)
    s = torch.tensor([scale])
    cache = mala.PagedCache(k, v, s.cuda(), s.cuda())
    mala.mala_paged_write(x.cuda(), x.cuda(), cuda(np.arange(512)), cache)
    want = pu.e4m3_of(x, s[:, None, None]).view(torch.uint8).view(32, 1, 16, 128)
    for t in (k, v):
        got = pu.raw(t).cpu()
        nan = (want & 0x7F) == 0x7F
        assert ((got & 0x7F) == 0x7F)[nan].all()
        assert torch.equal(got[~nan], want[~nan])
    pu.raw(k).copy_(torch.arange(256, dtype=torch.uint8).repeat(256).view(32, 1, 16, 128).cuda())
    out = mala.paged_read(cache, cuda(np.arange(32)[None]), cuda([0, 512]), 512, 512)["k"].cpu()
    b = torch.arange(256, dtype=torch.uint8).repeat(256).view(torch.float8_e4m3fn).float()
    want = (b * s).to(torch.bfloat16).view(1, 512, 128)
    nan = want.isnan()
    assert out.isnan()[nan].all() and torch.equal(out[~nan].view(torch.int16), want[~nan].view(torch.int16))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hkv,D,P,layout,lens", [
    (2, 128, 16, "hpd", [1]), (1, 64, 48, "phd", [0, 17, 0, 0, 300, 48, 0]),
    (8, 128, 32, "wide", [64, 1, 700, 33]), (3, 64, 64, "hpd", [5] * 300)])
def test_read(Hkv, D, P, layout, lens, e4m3):
    scales = dict(ks=np.linspace(0.5, 1.25, Hkv), vs=np.linspace(1.5, 0.75, Hkv)) if e4m3 else {}
    w = Batch(21, lens, Hkv, Hkv, D, P, e4m3, layout, **scales)
    cu = np.concatenate([[0], np.cumsum(lens)]) + 3      # rows before and behind are nobody's
    total = int(cu[-1]) + 9
    if max(lens) > 40:                                   # a missing page reads as zeros
        b = int(np.argmax(lens))
        w.table[b, 0] = -1
        w.k[b][:, :P], w.v[b][:, :P] = 0, 0
    k = torch.full((Hkv, total, D), 7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, -7.0)
    mala.mala_paged_read(w.cache, cuda(w.table), cuda(cu), max(lens), k, v)
    for got, rows, s, rest in ((k, w.k, w.ks, 7.0), (v, w.v, w.vs, -7.0)):
        want = torch.full((Hkv, total, D), rest, dtype=torch.float64)
        for b, n in enumerate(lens):
            x = rows[b] if s is None else (rows[b].float() * s[:, None, None]).double()
            want[:, cu[b]:cu[b] + n] = x
        assert torch.equal(got.cpu(), want.to(torch.bfloat16))
    # runs longer than max_seqlen are cut, the rows behind stay
    if max(lens) > 40:
        k.fill_(7.0)
        mala.mala_paged_read(w.cache, cuda(w.table), cuda(cu), 40, k, v)
        b = int(np.argmax(lens))
        assert (k[:, cu[b] + 40:cu[b] + lens[b]] == 7.0).all()
        assert (k[:, cu[b]:cu[b] + min(P, 40)] == 0.0).all()


# ------------------------------------------------------------------ together, as a server does
def _dense(q, k, v, scale):
    """Causal attention of the last rows in 64 bits: q [Hq, m, D], k, v [Hkv, n, D]."""
    g, m, n = q.shape[0] // k.shape[0], q.shape[1], k.shape[1]
    s = np.matmul(q, k.repeat(g, 0).transpose(0, 2, 1)) * scale
    s = np.where(np.arange(n) <= np.arange(m)[:, None] + n - m, s, -math.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    return np.matmul(p / p.sum(-1, keepdims=True), v.repeat(g, 0))


@pytest.mark.parametrize("D,P,e4m3", [(128, 16, False), (64, 48, True)])
def test_serving_run(D, P, e4m3):
    # requests come, are prefilled in chunks against their cached pages, decode, and leave;
    # pages of finished ones are used again
    Hq, Hkv, R, N, W = 4, 2, 6, 24 if P == 16 else 9, 20
    rng = np.random.default_rng(D)
    k, v = pu.pool(N, Hkv, P, D, e4m3)
    cache = mala.PagedCache(k, v)
    table = torch.full((R, W), -1, dtype=I32, device="cuda")
    ring, state = cuda(rng.permutation(N)), cuda([0, N])
    lens = torch.zeros(R, dtype=I32, device="cuda")
    hist = [[np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0, D))] for _ in range(R)]
    goal = [0] * R
    scale = float(np.float32(D ** -0.5))
    refused_once = False
    for step in range(14):
        have = [h[0].shape[1] for h in hist]
        new = []
        for r in range(R):
            if have[r] == 0:
                goal[r] = int(rng.integers(20, 150)) if rng.random() < 0.7 else 0
                new.append(min(goal[r], 70))
            elif have[r] < goal[r]:
                new.append(min(goal[r], have[r] + 70))
            else:
                new.append(0 if rng.random() < 0.2 else have[r] + 1)
        T = sum(max(0, a - b) for a, b in zip(new, have))
        out = mala.paged_update(lens, cuda(new), table, ring, state, T + 5, P, N)
        refused_once |= int(out["free_state"][2]) > 0
        lens, state, cu = out["lens"], out["free_state"], out["cu_seqlens"].cpu().numpy()
        got_lens = lens.cpu().numpy()
        kn, vn = pu.quarters(rng, (Hkv, T + 5, D)), pu.quarters(rng, (Hkv, T + 5, D))
        q = pu.quarters(rng, (Hq, T + 5, D), 4)
        mala.mala_paged_write(kn.to(torch.bfloat16).cuda(), vn.to(torch.bfloat16).cuda(),
                              out["slots"], cache)
        for r in range(R):
            if got_lens[r] == 0:
                hist[r] = [np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0, D))]
            elif got_lens[r] > have[r]:
                rows = slice(cu[r], cu[r + 1])
                hist[r] = [np.concatenate([hist[r][0], kn[:, rows].numpy()], 1),
                           np.concatenate([hist[r][1], vn[:, rows].numpy()], 1)]
            assert hist[r][0].shape[1] == got_lens[r]
        # decode of every request's last token (those without tokens have empty caches)
        longest = max(int(got_lens.max()), 1)
        qd = pu.quarters(rng, (R, Hq, D), 4)
        dec = mala.paged_decode(qd.to(torch.bfloat16).cuda(), cache, table, lens, longest, scale, 0.0)
        smax = scale * 2 * float(qd.abs().sum(2).max())
        to, _ = pu.decode_bounds(longest, smax, 2.0, False)
        for r in range(R):
            if got_lens[r] == 0:
                assert (dec["o"][r] == 0).all()
                continue
            want = _dense(qd[r].numpy()[:, None], *hist[r], scale)[:, 0]
            assert np.abs(dec["o"][r].double().cpu().numpy() - want).max() <= to
        # prefill of the grown requests' new tokens against their cached keys
        rows = [r for r in range(R) if got_lens[r] > have[r]]
        if not rows:
            continue
        nq = [int(got_lens[r]) - have[r] for r in rows]
        nk = [int(got_lens[r]) for r in rows]
        cq, ck = np.concatenate([[0], np.cumsum(nq)]), np.concatenate([[0], np.cumsum(nk)])
        kv = mala.paged_read(cache, table[rows].contiguous(), cuda(ck), max(nk), int(ck[-1]))
        qp = torch.cat([q[:, cu[r]:cu[r + 1]] for r in rows], 1)
        f = mala.fwd_varlen(qp.to(torch.bfloat16).cuda(), kv["k"], kv["v"], cuda(cq), max(nq), scale,
                            0.0, cu_seqlens_k=cuda(ck), max_seqlen_k=max(nk))
        for i, r in enumerate(rows):
            want = _dense(qp[:, cq[i]:cq[i + 1]].numpy(), *hist[r], scale)
            got = f["o"][:, cq[i]:cq[i + 1]].double().cpu().numpy()
            assert np.abs(got - want).max() <= 1e-2      # the forward's own bound
    used = sum(pu.pages_of(int(n), P) for n in lens.cpu())
    assert int(state[1]) + used == N
    assert refused_once


def test_step_captured_in_a_graph():
    # update, write and decode of one step in a graph, replayed for the steps of a batch with
    # eager work between the replays; the same steps eagerly give the same bits
    Hq, Hkv, D, P, R, N, W = 8, 2, 128, 16, 4, 64, 12
    rng = np.random.default_rng(31)
    start = [5, 31, 0, 64]

    def fresh():
        k, v = pu.pool(N, Hkv, P, D)
        t = dict(cache=mala.PagedCache(k, v), table=torch.full((R, W), -1, dtype=I32, device="cuda"),
                 ring=cuda(np.arange(N)), state=cuda([0, N, 0, 0]), lens=cuda([0] * R),
                 new=cuda(start), kn=torch.zeros((Hkv, 128, D), dtype=torch.bfloat16, device="cuda"),
                 q=torch.zeros((R, Hq, D), dtype=torch.bfloat16, device="cuda"))
        t["vn"] = t["kn"].clone()
        e = lambda *s: torch.zeros(s, dtype=I32, device="cuda")
        t.update(lens_out=e(R), cu=e(R + 1), slots=e(128), pos=e(128), state_out=e(4),
                 o=torch.zeros((R, Hq, D), device="cuda"), lse=torch.zeros((R, Hq), device="cuda"))
        need = mala.mala_paged_decode_workspace_size(R, Hq, Hkv, D, W * P, 32)
        t["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
        return t

    def step(t):
        mala.mala_paged_update(t["lens"], t["new"], t["table"], t["ring"], t["state"], t["lens_out"],
                               t["cu"], t["slots"], t["pos"], t["state_out"], P, N)
        mala.mala_paged_write(t["kn"], t["vn"], t["slots"], t["cache"])
        mala.mala_paged_decode(t["q"], t["cache"], t["table"], t["lens_out"], W * P, t["o"], t["lse"],
                               None, None, 32, t["ws"], 0.1, 0.0)
        t["lens"].copy_(t["lens_out"])
        t["state"].copy_(t["state_out"])

    eager, graphed = fresh(), fresh()
    warm = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graphed)
    for i in range(6):
        new = start if i == 0 else [n + (i if r != 2 else 9 * i) for r, n in enumerate(start)]
        kn = torch.from_numpy(rng.standard_normal((2, Hkv, 128, D))).to(torch.bfloat16)
        q = torch.from_numpy(rng.standard_normal((R, Hq, D))).to(torch.bfloat16)
        for t in (eager, graphed):
            t["new"].copy_(cuda(new))
            t["kn"].copy_(kn[0])
            t["vn"].copy_(kn[1])
            t["q"].copy_(q)
        step(eager)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for name in ("table", "ring", "lens", "cu", "slots", "pos", "state", "o", "lse"):
            assert torch.equal(eager[name], graphed[name]), (i, name)
        assert torch.equal(eager["cache"].k_pages, graphed["cache"].k_pages)
        assert eager["lens"].tolist() == new


def test_two_streams_at_once():
    # independent caches, workspaces and outputs on two streams give the sequential bits
    ws = [Batch(41 + i, [900, 300, 64], 8, 2, 128, 16) for i in range(2)]
    alone = [w.decode(split=64) for w in ws]
    streams = [torch.cuda.Stream() for _ in ws]
    args = [(w.q.to(torch.bfloat16).cuda(), cuda(w.table), cuda(w.lens)) for w in ws]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [mala.paged_decode(q, w.cache, t, n, 900, w.scale, 0.0, 64, stream=s)
               for w, s, (q, t, n) in zip(ws, streams, args)]
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])
