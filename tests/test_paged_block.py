"""The paged cache with a scale per block of 16 rows and head on the GPU against plain 64-bit forms:
writes with and without the rotation, reads, the decode, and a serving run of them together."""
import math

import numpy as np
import pytest
import torch

import block_util as bu
import paged_util as pu
import paper_2609_32712_amd as mala

pytestmark = pytest.mark.gpu

I32, BF16 = torch.int32, torch.bfloat16


def cuda(a, dtype=I32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def new_rows(x, order):
    """x [2, Hkv, T, D] bf16 (CPU) as k_new, v_new on the GPU."""
    if order == "heads":
        return x[0].cuda(), x[1].cuda()
    both = x.permute(2, 0, 1, 3).contiguous().cuda()      # slices of one [T, 2, Hkv, D] projection
    return both[:, 0].transpose(0, 1), both[:, 1].transpose(0, 1)


def snapshot(t, s):
    """(values float64 [N, H, P, D], e int64 [N, H, P / 16]) of a cache's tensors."""
    v = pu.raw(t).cpu().contiguous().view(torch.float8_e4m3fn).float().double().numpy()
    return v, s.view(torch.uint8).cpu().numpy().astype(np.int64) - 127


def check_cache(k, v, ks, vs, want):
    for t, s, (values, e) in ((k, ks, want[0]), (v, vs, want[1])):
        np.testing.assert_array_equal(s.view(torch.uint8).cpu().numpy().astype(np.int64) - 127, e)
        assert bu.same_bytes(pu.raw(t).cpu().contiguous(), bu.as_bytes(values))


class Cache:
    """A block-scaled cache on the GPU and its plain form, written side by side."""

    def __init__(self, seed, N, Hkv, P, D, layout="hpd", spread=6):
        self.rng = np.random.default_rng(seed)
        self.cache, self.k, self.v, self.ks, self.vs = bu.block_cache(mala, N, Hkv, P, D, layout)
        self.N, self.Hkv, self.P, self.D, self.spread = N, Hkv, P, D, spread
        # every byte but NaN and every scale, in range or not, may be there before
        for t, s in ((self.k, self.ks), (self.v, self.vs)):
            x = self.rng.integers(0, 256, t.shape).astype(np.uint8)
            x[(x & 0x7F) == 0x7F] = 0x7E
            pu.raw(t).copy_(torch.from_numpy(x).cuda())
            e = np.where(self.rng.random(s.shape) < 0.1, self.rng.integers(0, 256, s.shape),
                         self.rng.integers(118, 126, s.shape))
            s.view(torch.uint8).copy_(torch.from_numpy(e.astype(np.uint8)).cuda())
        self.plain = [snapshot(self.k, self.ks), snapshot(self.v, self.vs)]

    def rows(self, T):
        """[2, Hkv, T, D] bf16 normals, each token's of its own size."""
        x = self.rng.standard_normal((2, self.Hkv, T, self.D))
        x *= np.exp2(self.rng.uniform(-self.spread, self.spread, (2, self.Hkv, T, 1)))
        return torch.from_numpy(x).to(BF16)

    def write(self, slots, x=None, order="heads"):
        x = self.rows(len(slots)) if x is None else x
        kn, vn = new_rows(x, order)
        mala.mala_paged_write(kn, vn, cuda(slots), self.cache)
        for i in range(2):
            bu.write_plain(*self.plain[i], x[i].double().numpy(), slots)
        self.check()

    def check(self):
        check_cache(self.k, self.v, self.ks, self.vs, self.plain)


SHAPES = [(1, 64, 16, "hpd", "heads"), (2, 128, 16, "hpd", "tokens"), (5, 64, 48, "phd", "tokens"),
          (8, 128, 32, "wide", "heads"), (3, 128, 64, "phd", "heads"), (17, 64, 16, "hpd", "tokens")]


# ------------------------------------------------------------------ writes
@pytest.mark.parametrize("Hkv,D,P,layout,order", SHAPES)
def test_write_runs(Hkv, D, P, layout, order):
    # runs of consecutive slots that start and end anywhere in their blocks, padded, then appended to
    N = 60
    c = Cache(Hkv * D + P, N, Hkv, P, D, layout)
    for T in (1, 2, 16, 17, 40, 300):
        pages = c.rng.permutation(N)
        start = int(c.rng.integers(0, P))
        at = start + np.arange(T)
        slots = pages[at // P % N] * P + at % P
        slots = np.concatenate([slots, np.full(int(c.rng.integers(0, 70)), -1)])
        c.write(slots, order=order)
        c.write([int(slots[T - 1]) // 16 * 16 + (int(slots[T - 1]) + 1) % 16], order=order)


@pytest.mark.parametrize("T", [1, 63, 64, 1000, 2100])
def test_write_decodes(T):
    # a token for each of many blocks, at any row of it: the chunks of the launch are small and large
    c = Cache(T, T + 5, 2, 16, 64)
    for _ in range(3):
        slots = c.rng.permutation(T + 5)[:T] * 16 + c.rng.integers(0, 16, T)
        slots[c.rng.random(T) < 0.1] = -1
        c.write(slots)


def test_write_prompts_of_many_chunks():
    # as many tokens as fill the largest chunks, requests one after the other, and padding among them
    c = Cache(7, 2500, 1, 16, 64)
    parts, first = [], 0
    for n in c.rng.integers(1, 900, 80):
        if first + int(n) // 16 + 3 > 2500:
            break
        a = int(c.rng.integers(0, 16))
        parts.append(first * 16 + a + np.arange(n))
        parts.append(np.full(int(c.rng.integers(0, 4)), -1))
        first += (a + int(n)) // 16 + 1
    slots = np.concatenate(parts)
    assert len(slots) > 32768
    c.write(slots)


def test_write_windows_of_64_tokens():
    # the tokens of a block as far apart as they may be, blocks between each other, in any order
    c = Cache(3, 40, 2, 16, 128)
    slots = np.full(200, -1)
    slots[[0, 63]] = [5 * 16 + 3, 5 * 16 + 4]          # 64 consecutive tokens, first and last
    slots[[1, 40, 64]] = [6 * 16, 6 * 16 + 9, 6 * 16 + 1]
    slots[100:132] = c.rng.permutation(32) + 8 * 16    # two blocks in any order
    slots[[140, 150, 160, 170]] = [20 * 16 + 15, 21 * 16, 20 * 16, 21 * 16 + 15]
    c.write(slots)
    c.write(np.concatenate([np.full(77, -1), slots]))


def test_write_skips_slots_outside():
    c = Cache(4, 6, 2, 32, 64)
    c.write([-1, 6 * 32, 2 ** 31 - 1, -2 ** 31, 17, 5 * 32 + 31, -5, 18])
    c.write([-1, -1])
    c.write([])


def test_write_the_same_slot_twice_keeps_one_of_them():
    c = Cache(5, 4, 2, 16, 64)
    x = c.rows(6)
    slots = [16, 17, 17, 17, 18, 16]
    kn, vn = new_rows(x, "heads")
    before = [(a.copy(), e.copy()) for a, e in c.plain]
    mala.mala_paged_write(kn, vn, cuda(slots), c.cache)
    # each row holds one of the tokens that were sent to it, under the scale of those that stayed
    fits = 0
    for a in (0, 5):
        for b in (1, 2, 3):
            pick = [(p.copy(), e.copy()) for p, e in before]
            for i in range(2):
                bu.write_plain(*pick[i], x[i][:, [a, b, 4]].double().numpy(), [16, 17, 18])
            try:
                check_cache(c.k, c.v, c.ks, c.vs, pick)
                fits += 1
            except AssertionError:
                pass
    assert fits == 1


def test_write_scales_at_their_ends():
    # zeros, the smallest and the largest bf16, infinities and NaN; then growth over the whole range
    big, inf, nan = float(torch.finfo(BF16).max), math.inf, math.nan
    specials = [0.0, -0.0, 2.0 ** -133, 2.0 ** -126, 2.0 ** -127 * 1.5, 2.0 ** -118, 448.0 * 2.0 ** -117, big, -big,
                inf, -inf, nan, 448.0, 450.0, 1.0, 2.0 ** 120 * 240, 2.0 ** 127 * 1.75, 2.0 ** 120]
    c = Cache(6, 40, 2, 16, 64, spread=0)
    for i, s in enumerate(specials):
        x = torch.zeros((2, 2, 2, 64)).to(BF16)
        x[..., 0, :5] = torch.tensor([s, -s, 0.0, nan, s / 2]).to(BF16)
        x[..., 1, :3] = torch.tensor([inf, 1e-3 * s if math.isfinite(s) else 0.0, 0.0]).to(BF16)
        c.write([16 * i, 16 * i + 7], x)
        # (a larger row later: the rest of the block is rounded again, from any e to any other)
        y = torch.zeros((2, 2, 1, 64)).to(BF16)
        y[..., 5] = float(2.0 ** c.rng.integers(-126, 127))
        c.write([16 * i + 9], y)
    k = bu.held(c.k, c.ks)
    assert not np.isinf(k).any()


@pytest.mark.parametrize("first", [0.0, 2.0 ** -110, 3e-5, 1.0, 1e6])
def test_every_bf16(first):
    # all 65536 bf16 values in blocks of their own neighbours, on their own and behind a first row
    x = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(BF16).view(1, 512, 128)
    x = torch.stack([x, x.flip(1)])
    c = Cache(8, 40, 1, 16, 128)
    c.write(np.arange(16 * 32), x)
    row = torch.full((2, 1, 32, 128), first).to(BF16)
    c.write(np.arange(32) * 16, row)
    keep = torch.ones(512, dtype=torch.bool)
    keep[::16] = False
    c.write(np.arange(512)[keep.numpy()], x[:, :, keep])


def test_write_growth_keeps_the_error_of_two_roundings():
    # rows appended one by one, each larger: every row is within half a step of each scale it had
    c = Cache(9, 2, 1, 16, 64, spread=0)
    rows = [torch.from_numpy(c.rng.standard_normal((2, 1, 1, 64)) * 1.7 ** i).to(BF16) for i in range(16)]
    for i, x in enumerate(rows):
        c.write([16 + i], x)
    got, e = bu.held(c.k, c.ks)[1, 0], int(c.ks.view(torch.uint8)[1, 0, 0]) - 127
    for i, x in enumerate(rows):
        x = x[0, 0, 0].double().numpy()
        # normal values keep their first rounding (2^-4); below, half of 2^-9 of the scale, at each of
        # the scales: they double at least, so a whole one at most
        assert (np.abs(got[i] - x) <= 2.0 ** -4 * np.abs(x) * 1.0000001 + 2.0 ** -9 * 2.0 ** e).all()


# ------------------------------------------------------------------ the rotated write
@pytest.mark.parametrize("Hkv,D,P,layout,order", SHAPES)
@pytest.mark.parametrize("kind", ["block", "e4m3", "bf16"])
def test_rope_write_is_rope_and_write(Hkv, D, P, layout, order, kind):
    rng = np.random.default_rng(Hkv + D)
    N, group = 40, 3
    for T, R, lay, scale in ((1, D, 0, 1.0), (33, D // 2, 1, 1.25), (500, D - 16, 0, 0.5), (80, 16, 0, 1.0),
                             (1500, D, 1, 1.0)):
        if T > N * P:
            continue
        f, _ = mala.rope_frequencies(R, device="cuda")
        pos = torch.from_numpy(rng.integers(0, 100000, T)).int().cuda()
        start = int(rng.integers(0, P))
        at = (start + np.arange(T)) % (N * P)
        slots = rng.permutation(N)[at // P] * P + at % P
        if T == 80:
            slots[60:] = -1
        x = torch.from_numpy(rng.standard_normal((2, Hkv, T, D))).to(BF16)
        kn, vn = new_rows(x, order)
        q = torch.from_numpy(rng.standard_normal((T, Hkv * group, D))).to(BF16).cuda().transpose(0, 1)
        caches = []
        for _ in range(2):
            if kind == "block":
                one = bu.block_cache(mala, N, Hkv, P, D, layout, fill=0x31)
            else:
                k, v = pu.pool(N, Hkv, P, D, kind == "e4m3", layout)
                s = torch.linspace(0.01, 0.02, Hkv).cuda() if kind == "e4m3" else None
                one = (mala.PagedCache(k, v, s, s), k, v, None, None)
            caches.append(one)
        sep = mala.rope(q, kn, pos, f, lay, scale)
        mala.mala_paged_write(sep["k"], vn if vn.is_contiguous() else vn.contiguous(), cuda(slots), caches[0][0])
        for tokens_first in (True, False):
            got = mala.paged_rope_write(q, kn, vn, pos, cuda(slots), caches[1][0], f, lay, scale, tokens_first)
            assert got["q"].is_contiguous()
            assert torch.equal(got["q"].transpose(0, 1) if tokens_first else got["q"], sep["q"])
            for a, b in zip(caches[0][1:], caches[1][1:]):
                if a is not None:
                    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        # without queries, and in place
        mala.mala_paged_rope_write(None, None, kn, vn, pos, cuda(slots), caches[1][0], f, lay, scale)
        qi = q.clone()
        mala.mala_paged_rope_write(qi, qi, kn, vn, pos, cuda(slots), caches[1][0], f, lay, scale)
        assert torch.equal(qi, sep["q"])
        for a, b in zip(caches[0][1:], caches[1][1:]):
            if a is not None:
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("R", [16, 48, 64])
@pytest.mark.parametrize("T", [300, 1300, 2400, 3900, 4700])
def test_rope_write_of_many_decodes(T, R):
    # tokens alone in their blocks, one to sixteen of them to a workgroup: angles of as many rows
    rng = np.random.default_rng(T)
    f, _ = mala.rope_frequencies(R, device="cuda")
    pos = torch.from_numpy(rng.integers(0, 100000, T)).int().cuda()
    slots = rng.permutation(T) * 16 + rng.integers(0, 16, T)
    slots[rng.random(T) < 0.05] = -1
    kn, vn = new_rows(torch.from_numpy(rng.standard_normal((2, 2, T, 64))).to(BF16), "tokens")
    caches = [bu.block_cache(mala, T, 2, 16, 64, fill=0x75) for _ in range(2)]
    sep = mala.rope(kn, None, pos, f)["q"]
    mala.mala_paged_write(sep, vn.contiguous(), cuda(slots), caches[0][0])
    mala.mala_paged_rope_write(None, None, kn, vn, pos, cuda(slots), caches[1][0], f)
    for a, b in zip(caches[0][1:], caches[1][1:]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


# ------------------------------------------------------------------ reads
def test_read_of_every_byte_and_scale_is_exact():
    # 256 bytes x 256 scales: e4m3 x 2^e as a bf16, no rounding (bytes outside the range: its ends)
    cache, k, v, ks, vs = bu.block_cache(mala, 512, 1, 16, 128)
    pu.raw(k).copy_(torch.arange(256, dtype=torch.uint8).repeat(512 * 8).view(512, 1, 16, 128).cuda())
    pu.raw(v).copy_(pu.raw(k).flip(3))
    e = torch.arange(256, dtype=torch.int32).repeat(2)
    ks.view(torch.uint8).copy_(e.to(torch.uint8).view(512, 1, 1).cuda())
    vs.view(torch.uint8).copy_(e.flip(0).to(torch.uint8).view(512, 1, 1).cuda())
    out = mala.paged_read(cache, cuda(np.arange(512)[None]), cuda([0, 8192]), 8192, 8192)
    for t, s, got in ((k, ks, out["k"]), (v, vs, out["v"])):
        x = pu.raw(t).cpu().view(torch.float8_e4m3fn).float().double()
        p = torch.exp2((s.view(torch.uint8).cpu().double() - 127).clamp(-117, 120))
        want = (x * p[..., None]).view(1, 8192, 128).to(BF16)
        got, nan = got.cpu(), want.isnan()
        fine = want.isfinite()
        # (a bf16 but for 256 .. 448 x 2^120, which no write makes)
        assert torch.equal(want[fine].double(), (x * p[..., None]).view(1, 8192, 128)[fine])
        assert got.isnan()[nan].all()
        assert torch.equal(got[~nan].view(torch.int16), want[~nan].view(torch.int16))


@pytest.mark.parametrize("Hkv,D,P,layout,lens", [
    (2, 128, 16, "hpd", [1]), (1, 64, 48, "phd", [0, 17, 0, 0, 300, 48, 0]),
    (8, 128, 32, "wide", [64, 1, 700, 33]), (3, 64, 64, "hpd", [5] * 300)])
def test_read(Hkv, D, P, layout, lens):
    w = Batch(21, lens, Hkv, Hkv, D, P, layout)
    cu = np.concatenate([[0], np.cumsum(lens)]) + 3      # rows before and behind are nobody's
    total = int(cu[-1]) + 9
    if max(lens) > 40:                                   # a missing page reads as zeros
        b = int(np.argmax(lens))
        w.table[b, 0] = -1
        w.k[b][:, :P], w.v[b][:, :P] = 0, 0
    k = torch.full((Hkv, total, D), 7.0, dtype=BF16, device="cuda")
    v = torch.full_like(k, -7.0)
    mala.mala_paged_read(w.cache, cuda(w.table), cuda(cu), max(lens), k, v)
    for got, rows, rest in ((k, w.k, 7.0), (v, w.v, -7.0)):
        want = torch.full((Hkv, total, D), rest, dtype=torch.float64)
        for b, n in enumerate(lens):
            want[:, cu[b]:cu[b] + n] = rows[b]
        assert torch.equal(got.cpu().double(), want)


# ------------------------------------------------------------------ decode
class Batch:
    """Sequences in scattered pages: quarters (see paged_util) times 2^e, e of each block in
    [-1, 1]; products of q and K are multiples of 1/32 and sums of 128 of them exact in fp32.  Rows
    that are not valid hold NaN, and blocks without a valid row a scale of NaN."""

    def __init__(self, seed, lens, Hq, Hkv, D, P, layout="hpd", needle=0.0, width=None):
        rng = np.random.default_rng(seed)
        self.rng, self.lens, self.Hq, self.Hkv, self.D, self.P = rng, lens, Hq, Hkv, D, P
        self.table, self.N = pu.scatter_tables(rng, lens, P, width=width)
        raw = [[pu.quarters(rng, (Hkv, n, D)) for n in lens] for _ in range(2)]
        self.cache, k, v, ks, vs = bu.block_cache(mala, self.N, Hkv, P, D, layout, fill=0x7F)
        ks.view(torch.uint8).fill_(255)
        vs.view(torch.uint8).fill_(255)
        self.k, self.v = [], []
        for t, s, rows, mine in ((k, ks, raw[0], self.k), (v, vs, raw[1], self.v)):
            pu.fill(t, self.table, lens, rows, P)
            scales = np.full((self.N, Hkv, P // 16), 255, np.uint8)
            for b, n in enumerate(lens):
                e = rng.integers(-1, 2, (Hkv, -(-n // 16)))
                for j in range(-(-n // 16)):
                    scales[self.table[b, 16 * j // P], :, 16 * j % P // 16] = e[:, j] + 127
                mine.append(rows[b] * torch.from_numpy(np.exp2(np.repeat(e, 16, 1)[:, :n, None].astype(float))))
            s.view(torch.uint8).copy_(torch.from_numpy(scales).cuda())
        self.q = pu.quarters(rng, (len(lens), Hq, D), 4)
        if needle:
            for b, n in enumerate(lens):
                for h in range(Hq if n else 0):
                    self.q[b, h] = self.q[b, h] / 4 + needle * torch.sign(
                        self.k[b][h // (Hq // Hkv), rng.integers(n)])
            self.q = torch.round(self.q * 4) / 4
        self.scale = float(np.float32(D ** -0.5))

    def seen(self, b):
        p = self.table[b, np.arange(self.lens[b]) // self.P]
        return (p >= 0) & (p < self.N)

    def plain(self, tau=0.0, split=256):
        return [pu.decode_seq(self.q[b].numpy(), self.k[b].numpy(), self.v[b].numpy(), self.seen(b),
                              self.scale, tau, split, n) for b, n in enumerate(self.lens)]

    def decode(self, tau=0.0, split=256, max_len=None, **kw):
        return mala.paged_decode(self.q.to(BF16).cuda(), self.cache, cuda(self.table), cuda(self.lens),
                                 max_len or max(max(self.lens), 1), self.scale, tau, split_tokens=split, **kw)

    def check(self, got, want, out_bf16=False, clear=None):
        o, lse = got["o"].double().cpu().numpy(), got["lse"].double().cpu().numpy()
        for b, n in enumerate(self.lens):
            wo, wl = want[b][0], want[b][1]
            none = np.isneginf(wl)
            assert np.isneginf(lse[b][none]).all() and (o[b][none] == 0).all(), b
            skip = none if clear is None else none | ~clear[b]
            if skip.all():
                continue
            smax = self.scale * 4.0 * float(self.q[b].abs().sum(1).max())
            to, tl = pu.decode_bounds(n, smax, 4.0, out_bf16)
            assert np.abs(o[b] - wo)[~skip].max() <= to, (b, np.abs(o[b] - wo).max(), to)
            assert np.abs(lse[b] - wl)[~skip].max() <= tl, (b, np.abs(lse[b] - wl).max(), tl)


LENS = [1, 0, 15, 16, 17, 31, 32, 33, 100, 129, 255, 257, 700]
DENSE = [
    # Hq, Hkv, D, P, layout, split
    (4, 2, 128, 16, "hpd", 32), (8, 1, 64, 48, "phd", 256), (7, 1, 64, 16, "hpd", 128),
    (33, 1, 64, 256, "wide", 512), (32, 2, 128, 80, "phd", 160), (40, 2, 128, 64, "wide", 256)]


@pytest.mark.parametrize("Hq,Hkv,D,P,layout,split", DENSE)
def test_decode_dense(Hq, Hkv, D, P, layout, split):
    w = Batch(1, LENS, Hq, Hkv, D, P, layout)
    want = w.plain()
    for out in (torch.float32, BF16):
        got = w.decode(split=split, out_dtype=out)
        w.check(got, want, out == BF16)
        assert got["head_tiles"].cpu().numpy().tolist() == [x[2].tolist() for x in want]
    bare = w.decode(split=split, out_dtype=BF16, stats=False)
    assert torch.equal(bare["o"], got["o"]) and torch.equal(bare["lse"], got["lse"])


@pytest.mark.parametrize("B,n", [(1, 1), (1, 200), (1, 5000), (3, 2047), (40, 700), (300, 130)])
@pytest.mark.parametrize("D", [128, 64])
def test_decode_batches(B, n, D):
    # whole caches in a workgroup, many blocks of one, more blocks than CUs
    rng = np.random.default_rng(B)
    lens = [n] * B if B < 40 else [int(x) for x in rng.integers(0, n + 1, B)]
    w = Batch(2, lens, 8, 2, D, 16)
    w.check(w.decode(), w.plain())


@pytest.mark.parametrize("D,P,layout,split,lens", [
    (128, 16, "hpd", 32, LENS), (64, 48, "phd", 64, LENS), (128, 64, "wide", 256, LENS),
    (128, 16, "hpd", 128, [2000] * 40), (64, 32, "hpd", 128, [900] * 200)])
@pytest.mark.parametrize("tau", [0.05, 0.3])
def test_decode_rule(D, P, layout, split, lens, tau):
    # what is retained, by splits shared between the wavefronts and by a wavefront per split
    w = Batch(3, lens, 8, 2, D, P, layout, needle=1.0)
    want = w.plain(tau, split)
    # heads whose decisions are clear of ties by what the scores' and the sums' roundings can move
    smax = w.scale * 4 * float(w.q.abs().sum(2).max())
    clear = [x[4] > 250 * pu.U24 + 16 * pu.U24 * (smax + 1) for x in want]
    assert sum(x.sum() for x in clear) >= 0.9 * 8 * len(lens)
    got = w.decode(tau, split)
    w.check(got, want, clear=clear)
    tiles = got["head_tiles"].cpu().numpy()
    for b, x in enumerate(want):
        assert tiles[b][clear[b]].tolist() == x[2][clear[b]].tolist()
    if all(c.all() for c in clear):
        h = sum(pu.set_hash(x[3][i], b, i) for b, x in enumerate(want) for i in range(8)) & ((1 << 64) - 1)
        assert int(got["counters"][mala.CNT_SET_HASH]) & ((1 << 64) - 1) == h


@pytest.mark.parametrize("tau,split", [(0.0, 256), (0.1, 64)])
def test_decode_missing_pages(tau, split):
    # windows that have moved on, holes, entries outside the pool, a row without any page
    w = Batch(4, [300, 500, 40, 700], 8, 2, 128, 16, needle=1.0, width=50)
    w.table[0, :10] = -1
    w.table[1, 3], w.table[1, 7:9], w.table[1, -1] = w.N, 2 ** 31 - 1, 0
    w.table[2] = -1
    w.table[3, 1::2] = -2 ** 31
    want = w.plain(tau, split)
    smax = w.scale * 4 * float(w.q.abs().sum(2).max())
    clear = [x[4] > 250 * pu.U24 + 16 * pu.U24 * (smax + 1) for x in want]
    w.check(w.decode(tau, split), want, clear=clear)


def test_decode_does_not_depend_on_the_batch():
    lens = [700, 33, 512, 1]
    w = Batch(11, lens, 8, 2, 128, 16, needle=1.0)
    for tau in (0.0, 0.1):
        whole = w.decode(tau, 128)
        q, t = w.q.to(BF16).cuda(), cuda(w.table)
        for b, n in enumerate(lens):
            one = mala.paged_decode(q[b:b + 1], w.cache, t[b:b + 1], cuda([n]), 700, w.scale, tau, 128)
            assert torch.equal(one["head_tiles"][0], whole["head_tiles"][b])
            to, tl = pu.decode_bounds(700, 120.0, 4.0, False)
            assert (one["o"][0] - whole["o"][b]).abs().max() <= 2 * to
            assert (one["lse"][0] - whole["lse"][b]).abs().max() <= 2 * tl


def test_decode_is_the_bf16_caches_of_the_same_values():
    # the values of the blocks, cached as bf16: the same products and the same sums
    w = Batch(12, [900, 47, 333], 8, 2, 128, 16, needle=1.0)
    k, v = pu.pool(w.N, 2, 16, 128)
    pu.fill(k, w.table, w.lens, w.k, 16)
    pu.fill(v, w.table, w.lens, w.v, 16)
    other = mala.PagedCache(k, v)
    for tau in (0.0, 0.1):
        a = w.decode(tau, 64)
        b = mala.paged_decode(w.q.to(BF16).cuda(), other, cuda(w.table), cuda(w.lens), 900, w.scale, tau, 64)
        assert torch.equal(a["head_tiles"], b["head_tiles"])
        to, tl = pu.decode_bounds(900, 120.0, 4.0, False)
        assert (a["o"] - b["o"]).abs().max() <= 2 * to and (a["lse"] - b["lse"]).abs().max() <= 2 * tl


def test_decode_of_far_scales_and_long_offsets():
    # scales of 2^-60 on K with queries of 2^60, values of 2^100; the pool's end past 2^32 bytes
    P, D, N = 256, 128, 70000
    cache, k, v, ks, vs = bu.block_cache(mala, N, 2, P, D)
    assert pu.raw(k).numel() > 2 ** 32
    table = cuda([[N - 1, 0, N - 2]])
    x = torch.from_numpy(np.random.default_rng(1).integers(-8, 9, (2, 2, 700, D)) / 4.0)
    kn = (x[0] * 2.0 ** -60).to(BF16).cuda()
    vn = (x[1] * 2.0 ** 100).to(BF16).cuda()
    at = np.arange(700)
    slots = np.array([N - 1, 0, N - 2])[at // P] * P + at % P
    mala.mala_paged_write(kn, vn, cuda(slots), cache)
    q = torch.from_numpy(np.random.default_rng(2).integers(-4, 5, (1, 4, D)) / 4.0)
    got = mala.paged_decode((q * 2.0 ** 60).to(BF16).cuda(), cache, table, cuda([700]), 700, 0.125, 0.0)
    o, lse, _, _, _ = pu.decode_seq(q[0].numpy(), x[0].numpy(), x[1].numpy(), np.ones(700, bool), 0.125, 0.0, 256,
                                    700)
    to, tl = pu.decode_bounds(700, 0.125 * 2 * float(q.abs().sum(2).max()), 2.0, False)
    assert np.abs(got["o"][0].double().cpu().numpy() / 2.0 ** 100 - o).max() <= to
    assert np.abs(got["lse"][0].double().cpu().numpy() - lse).max() <= tl


# ------------------------------------------------------------------ together, as a server does
def _dense(q, k, v, scale):
    g, m, n = q.shape[0] // k.shape[0], q.shape[1], k.shape[1]
    s = np.matmul(q, k.repeat(g, 0).transpose(0, 2, 1)) * scale
    s = np.where(np.arange(n) <= np.arange(m)[:, None] + n - m, s, -math.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    return np.matmul(p / p.sum(-1, keepdims=True), v.repeat(g, 0))


@pytest.mark.parametrize("D,P,tokens", [(128, 16, True), (64, 48, False)])
def test_serving_run(D, P, tokens):
    # update -> rotated write -> read and prefill of the chunks -> decode, over a run in which requests
    # come, grow by chunks and tokens, are cut back, leave, and their pages are used again.  What the
    # cache has to hold is followed by the plain forms; the attention is dense attention over that.
    Hq, Hkv, R, N, W = 4, 2, 6, 24 if P == 16 else 9, 20
    rng = np.random.default_rng(D)
    cache, k, v, ks, vs = bu.block_cache(mala, N, Hkv, P, D, "phd", fill=0x7E)
    plain = [snapshot(k, ks), snapshot(v, vs)]
    table = torch.full((R, W), -1, dtype=I32, device="cuda")
    ring, state = cuda(rng.permutation(N)), cuda([0, N])
    lens = torch.zeros(R, dtype=I32, device="cuda")
    f, turn = mala.rope_frequencies(D, factor=2.0, scaling="yarn", original_len=64, device="cuda")
    scale = float(np.float32(D ** -0.5))
    goal = [0] * R
    for step in range(14):
        have = lens.tolist()
        new = []
        for r in range(R):
            if have[r] == 0:
                goal[r] = int(rng.integers(20, 150)) if rng.random() < 0.7 else 0
                new.append(min(goal[r], 70))
            elif have[r] < goal[r]:
                new.append(min(goal[r], have[r] + 70))
            else:
                new.append([0, max(0, have[r] - 5), have[r] + 1][int(rng.choice(3, p=[0.2, 0.1, 0.7]))])
        T = sum(max(0, a - b) for a, b in zip(new, have))
        out = mala.paged_update(lens, cuda(new), table, ring, state, T + 5, P, N)
        lens, state, cu = out["lens"], out["free_state"], out["cu_seqlens"].cpu().numpy()
        now = lens.tolist()
        x = torch.from_numpy(rng.standard_normal((2, Hkv, T + 5, D)) * 2.0 ** (step % 5)).to(BF16)
        q = torch.from_numpy(rng.standard_normal((T + 5, Hq, D))).to(BF16).cuda().transpose(0, 1)
        kn, vn = new_rows(x, "tokens" if tokens else "heads")
        got = mala.paged_rope_write(q, kn, vn, out["positions"], out["slots"], cache, f, scale=turn)
        keys = mala.rope(kn, None, out["positions"], f, scale=turn)["q"].double().cpu().numpy()
        slots = out["slots"].tolist()
        bu.write_plain(*plain[0], keys, slots)
        bu.write_plain(*plain[1], x[1].double().numpy(), slots)
        check_cache(k, v, ks, vs, plain)
        hk, hv = bu.held(k, ks), bu.held(v, vs)
        tab = table.cpu().numpy()

        def rows(pool, r):
            at = np.arange(now[r])
            return pool[tab[r, at // P], :, at % P].transpose(1, 0, 2)

        longest = max(max(now), 1)
        qd = torch.from_numpy(rng.standard_normal((R, Hq, D))).to(BF16)
        qt = mala.rope(qd.cuda().transpose(0, 1), None, (lens - 1).contiguous(), f, scale=turn)["q"]
        qt = qt.transpose(0, 1).contiguous()
        dec = mala.paged_decode(qt, cache, table, lens, longest, scale, 0.0)
        for r in range(R):
            if now[r] == 0:
                assert (dec["o"][r] == 0).all()
                continue
            kr, vr = rows(hk, r), rows(hv, r)
            qr = qt[r].double().cpu().numpy()
            want = _dense(qr[:, None], kr, vr, scale)[:, 0]
            # (scores here are rounded sums of D products: D + 3 half steps of sum |q k|)
            smax = scale * float((np.abs(qr).reshape(Hkv, -1, 1, D) * np.abs(kr)[:, None]).sum(-1).max())
            to, _ = pu.decode_bounds(now[r], smax, float(np.abs(vr).max()), False)
            to += 2 * (D + 3) * pu.U24 * smax * float(np.abs(vr).max())
            assert np.abs(dec["o"][r].double().cpu().numpy() - want).max() <= to
        # prefill of the grown requests' new tokens against their cached keys
        grown = [r for r in range(R) if now[r] > have[r]]
        if not grown:
            continue
        nq, nk = [now[r] - have[r] for r in grown], [now[r] for r in grown]
        cq, ck = np.concatenate([[0], np.cumsum(nq)]), np.concatenate([[0], np.cumsum(nk)])
        kv = mala.paged_read(cache, table[grown].contiguous(), cuda(ck), max(nk), int(ck[-1]))
        for i, r in enumerate(grown):
            assert (kv["k"][:, ck[i]:ck[i + 1]].double().cpu().numpy() == rows(hk, r)).all()
            assert (kv["v"][:, ck[i]:ck[i + 1]].double().cpu().numpy() == rows(hv, r)).all()
        qp = torch.cat([got["q"][:, cu[r]:cu[r + 1]] for r in grown], 1)
        fw = mala.fwd_varlen(qp, kv["k"], kv["v"], cuda(cq), max(nq), scale, 0.0, cu_seqlens_k=cuda(ck),
                             max_seqlen_k=max(nk))
        for i, r in enumerate(grown):
            want = _dense(qp[:, cq[i]:cq[i + 1]].double().cpu().numpy(), rows(hk, r), rows(hv, r), scale)
            got_o = fw["o"][:, cq[i]:cq[i + 1]].double().cpu().numpy()
            # P as two bf16 terms (2^-16), and the scores' sums as above
            vmax = float(np.abs(rows(hv, r)).max())
            smax = scale * float(qp.float().abs().sum(-1).max()) * float(np.abs(rows(hk, r)).max())
            assert np.abs(got_o - want).max() <= (2.0 ** -14 + (2 * D + 600) * pu.U24 * (smax + 1)) * vmax
    used = sum(pu.pages_of(int(n), P) for n in lens.cpu())
    assert int(state[1]) + used == N


def test_step_captured_in_a_graph():
    # update, rotated write and decode of a step in a graph, replayed with eager work between the
    # replays: the same bits as eagerly, the grown scales among them
    Hq, Hkv, D, P, R, N, W = 8, 2, 128, 16, 4, 64, 12
    rng = np.random.default_rng(31)
    start = [5, 31, 0, 64]
    f, _ = mala.rope_frequencies(D, device="cuda")

    def fresh():
        cache, k, v, ks, vs = bu.block_cache(mala, N, Hkv, P, D)
        t = dict(cache=cache, ks=ks, vs=vs, table=torch.full((R, W), -1, dtype=I32, device="cuda"),
                 ring=cuda(np.arange(N)), state=cuda([0, N, 0, 0]), lens=cuda([0] * R), new=cuda(start),
                 kn=torch.zeros((Hkv, 128, D), dtype=BF16, device="cuda"),
                 qn=torch.zeros((Hq, 128, D), dtype=BF16, device="cuda"),
                 q=torch.zeros((R, Hq, D), dtype=BF16, device="cuda"))
        t["vn"], t["qt"] = t["kn"].clone(), t["qn"].clone()
        e = lambda *s: torch.zeros(s, dtype=I32, device="cuda")
        t.update(lens_out=e(R), cu=e(R + 1), slots=e(128), pos=e(128), state_out=e(4),
                 o=torch.zeros((R, Hq, D), device="cuda"), lse=torch.zeros((R, Hq), device="cuda"))
        need = mala.mala_paged_decode_workspace_size(R, Hq, Hkv, D, W * P, 32)
        t["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
        return t

    def step(t):
        mala.mala_paged_update(t["lens"], t["new"], t["table"], t["ring"], t["state"], t["lens_out"],
                               t["cu"], t["slots"], t["pos"], t["state_out"], P, N)
        mala.mala_paged_rope_write(t["qn"], t["qt"], t["kn"], t["vn"], t["pos"], t["slots"], t["cache"], f)
        mala.mala_paged_decode(t["q"], t["cache"], t["table"], t["lens_out"], W * P, t["o"], t["lse"],
                               None, None, 32, t["ws"], 0.1, 0.0)
        t["lens"].copy_(t["lens_out"])
        t["state"].copy_(t["state_out"])

    eager, graphed, warm = fresh(), fresh(), fresh()
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
        x = torch.from_numpy(rng.standard_normal((2, Hkv, 128, D)) * 3.0 ** i).to(BF16)
        q = torch.from_numpy(rng.standard_normal((Hq, 128, D))).to(BF16)
        for t in (eager, graphed):
            t["new"].copy_(cuda(new))
            t["kn"].copy_(x[0])
            t["vn"].copy_(x[1])
            t["qn"].copy_(q)
            t["q"].copy_(q[:, :R].transpose(0, 1))
        step(eager)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for name in ("table", "ring", "lens", "cu", "slots", "pos", "state", "o", "lse", "qt"):
            assert torch.equal(eager[name], graphed[name]), (i, name)
        for name in ("ks", "vs"):
            assert torch.equal(eager[name].view(torch.uint8), graphed[name].view(torch.uint8))
        for a, b in ((eager["cache"].k_pages, graphed["cache"].k_pages),
                     (eager["cache"].v_pages, graphed["cache"].v_pages)):
            assert torch.equal(pu.raw(a), pu.raw(b))
        assert eager["lens"].tolist() == new


def test_two_streams_at_once():
    ws = [Batch(41 + i, [900, 300, 64], 8, 2, 128, 16) for i in range(2)]
    alone = [w.decode(split=64) for w in ws]
    streams = [torch.cuda.Stream() for _ in ws]
    args = [(w.q.to(BF16).cuda(), cuda(w.table), cuda(w.lens)) for w in ws]
    caches = [Cache(50 + i, 80, 2, 16, 64) for i in range(2)]
    slots = [np.arange(100, 300 + 50 * i) for i in range(2)]
    rows = [c.rows(len(s)) for c, s in zip(caches, slots)]
    new = [(*new_rows(x, "tokens"), cuda(s)) for x, s in zip(rows, slots)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [mala.paged_decode(q, w.cache, t, n, 900, w.scale, 0.0, 64, stream=s)
               for w, s, (q, t, n) in zip(ws, streams, args)]
        for c, s, (kn, vn, sl) in zip(caches, streams, new):
            mala.mala_paged_write(kn, vn, sl, c.cache, stream=s)
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])
    for c, x, s in zip(caches, rows, slots):
        for i in range(2):
            for _ in range(3):      # (the second and third write find the scales of the first)
                bu.write_plain(*c.plain[i], x[i].double().numpy(), list(s))
        c.check()


def test_refusals_of_the_binding():
    cache = bu.block_cache(mala, 4, 2, 32, 64)[0]
    f, _ = mala.rope_frequencies(64, device="cuda")
    x = torch.zeros((2, 5, 64), dtype=BF16, device="cuda")
    p, s = torch.zeros(5, dtype=I32, device="cuda"), torch.zeros(5, dtype=I32, device="cuda")
    good = (x, x.clone(), x, x, p, s, cache, f)
    mala.mala_paged_rope_write(*good)
    put = lambda i, y: good[:i] + (y,) + good[i + 1:]
    for err, args in ((TypeError, put(6, None)), (ValueError, put(1, None)), (ValueError, put(0, None)),
                      (ValueError, put(0, x[:, :4])), (TypeError, put(0, x.float())),
                      (TypeError, put(1, x.float())), (ValueError, put(2, x[:1])),
                      (TypeError, put(3, x.float())), (ValueError, put(4, p[:4])), (TypeError, put(4, p.long())),
                      (ValueError, put(5, s[:4])), (TypeError, put(7, f.float())),
                      (ValueError, put(4, torch.zeros((2, 5), dtype=I32, device="cuda"))),
                      (mala.MalaError, put(7, f[:12])), (TypeError, put(0, x.cpu())),
                      (TypeError, put(5, s.cpu()))):
        with pytest.raises(err):
            mala.mala_paged_rope_write(*args)
