"""What the paged decode's description promises beyond its formulas, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2609_32712_amd as mala
import paged_util as pu

pytestmark = pytest.mark.gpu


class Normals:
    """Sequences of `lens` over one pool of normal values, each of random pages of it (pages may
    be several sequences')."""

    def __init__(self, seed, lens, Hq, Hkv, D, P=16, e4m3=False, pages=512, q_scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.D, self.P, self.N = lens, Hq, Hkv, D, P, pages
        x = torch.randn((2, pages, Hkv, P, D), generator=g, device="cuda")
        x = x.to(torch.float8_e4m3fn if e4m3 else torch.bfloat16)
        self.cache = mala.PagedCache(x[0], x[1])
        W = max(1, max(pu.pages_of(n, P) for n in lens))
        self.table = torch.randint(pages, (len(lens), W), generator=g, device="cuda",
                                   dtype=torch.int32)
        self.q = (torch.randn((len(lens), Hq, D), generator=g, device="cuda") * q_scale).bfloat16()
        self.n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.scale = float(np.float32(D ** -0.5))

    def decode(self, tau, split, max_len=None, rows=slice(None), **kw):
        return mala.paged_decode(self.q[rows], self.cache, self.table[rows].contiguous(), self.n[rows],
                                 max_len or max(self.lens), self.scale, tau, split_tokens=split, **kw)


@pytest.mark.parametrize("lens,Hq,Hkv,D,e4m3,tau,split", [
    ([9000, 4000, 700, 33, 0], 32, 8, 128, False, 0.0, 256),      # joined and whole caches
    ([9000, 4000, 700, 33, 0], 32, 8, 64, True, 0.0, 256),
    ([9000, 4000, 700, 33, 0], 32, 8, 128, True, 1e-3, 128),      # a wavefront per split
    ([9000, 4000, 700, 33, 0], 32, 8, 64, False, 1e-3, 128),
    ([4000, 500, 1], 16, 4, 128, False, 1e-3, 256),               # splits shared by wavefronts
    ([200, 300] * 20, 40, 2, 64, False, 0.0, 256)])               # more than 16 heads, no join
def test_bf16_outputs_are_the_fp32_ones_rounded_once(lens, Hq, Hkv, D, e4m3, tau, split):
    w = Normals(1, lens, Hq, Hkv, D, e4m3=e4m3)
    full, half = (w.decode(tau, split, out_dtype=t) for t in (torch.float32, torch.bfloat16))
    assert torch.equal(half["o"], full["o"].to(torch.bfloat16))
    assert torch.equal(half["lse"], full["lse"])
    assert torch.equal(half["head_tiles"], full["head_tiles"])


def _near_ties(s, n, tau, split):
    """Tolerances at which some decision is a tie: of every head and split of scores s [Hq, n]
    (64 bits), the test value nearest to tau in the split's chain of decisions."""
    out = []
    for x in s:
        for lo in range(0, n, split):
            run, best = -np.inf, None
            for a in range(lo + (min(n, lo + split) - 1 - lo) // 32 * 32, lo - 1, -32):
                tile = x[a:min(a + 32, n)]
                T = np.inf if run == -np.inf else n * np.exp(tile.max() - run)
                if best is None or abs(np.log(T / tau)) < abs(np.log(best / tau)):
                    best = T
                if T >= tau:
                    run = np.logaddexp.reduce(np.append(tile, run))
            if np.isfinite(best):
                out.append(best)
    return out


@pytest.mark.parametrize("D,e4m3,split", [(128, False, 256), (64, True, 128), (128, True, 512)])
def test_retained_sets_do_not_depend_on_the_batch_at_ties(D, e4m3, split):
    # alone the sequence's splits are shared by wavefronts, in a batch of 70 of them each
    # wavefront takes its own: every decision has to be the same, those on the border of the
    # tolerance (to the last bit of it, and a few to either side) among them
    Hq, Hkv, n, tau = 8, 2, 2000, 0.05
    w = Normals(2, [n] * 70, Hq, Hkv, D, e4m3=e4m3, q_scale=2.0)
    w.q[1:], w.table[1:] = w.q[:1], w.table[:1]
    pos = np.arange(n)
    rows = w.cache.k_pages.float().double().cpu().numpy()[w.table[0].cpu().numpy()[pos // w.P], :, pos % w.P]
    q = w.q[0].double().cpu().numpy()
    s = np.stack([rows[:, h // (Hq // Hkv)] @ q[h] for h in range(Hq)]) * w.scale
    some = 0
    for t in _near_ties(s, n, tau, split):
        for t32 in np.float32(t) * (1 + np.arange(-2, 3, dtype=np.float32) * np.float32(2 ** -23)):
            alone = w.decode(float(t32), split, rows=slice(1))
            batch = w.decode(float(t32), split)
            tiles = batch["head_tiles"]
            assert (tiles == tiles[0]).all() and torch.equal(alone["head_tiles"][0], tiles[0]), t32
            some += int((tiles[0] < -(-n // 32)).any())
    assert some > 100


@pytest.mark.parametrize("tau", [1.0, 300.0])
@pytest.mark.parametrize("D", [64, 128])
def test_default_split_gives_a_request_the_same_tiles_in_every_batch(D, tau):
    # alone, beside others, and sized for longer caches (as a captured step is)
    w = Normals(3, [3000, 700, 8000] * 12, 16, 4, D, q_scale=2.0)
    call = lambda rows, n: mala.paged_decode(w.q[rows], w.cache, w.table[rows].contiguous(), w.n[rows], n,
                                             w.scale, tau)
    whole = call(slice(None), 8000)
    if tau > 1:       # (L = n: against splits of 128 keys of 8000 a test value is 60 and more)
        assert int(whole["counters"][mala.CNT_RETAINED]) < int(whole["counters"][mala.CNT_LEGAL])
    for b, n in enumerate(w.lens[:3]):
        for longest in (n, 8000):
            assert torch.equal(call(slice(b, b + 1), longest)["head_tiles"][0], whole["head_tiles"][b])


def test_a_windowed_request_leaves_and_its_pages_are_taken_again():
    # missing pages are no pages to give back: the caller puts the row's own on the ring and
    # passes length 0.  The next requests need every page of the pool, and get rows of their own.
    rng = np.random.default_rng(9)
    P, W, N, Hkv, Hq, D = 16, 8, 10, 2, 4, 64
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    k, v = pu.pool(N, Hkv, P, D)
    cache = mala.PagedCache(k, v)
    table = torch.full((3, W), -1, dtype=torch.int32, device="cuda")
    ring, state = i32(rng.permutation(N)), i32([7, N])
    step = mala.paged_update(i32([0, 0, 0]), i32([100, 48, 0]), table, ring, state, 160, P, N)
    lens, state = step["lens"], step["free_state"]
    assert lens.tolist() == [100, 48, 0] and state.tolist()[:3] == [7, 0, 0]

    def put(row, places):                 # own pages of a row: behind the last free one
        head, count = state.tolist()[:2]
        at = (head + count + torch.arange(len(places), device="cuda")) % N
        ring[at] = table[row, places]
        table[row, places] = -1
        state[1] += len(places)

    put(0, [0, 1, 2])                     # the window moves on by three pages
    put(0, [3, 4, 5, 6])                  # and the request leaves
    step = mala.paged_update(i32([0, 48, 0]), i32([0, 48, 112]), table, ring, state, 200, P, N)
    assert step["lens"].tolist() == [0, 48, 112] and int(step["free_state"][2]) == 0
    lens, state, cu = step["lens"].tolist(), step["free_state"].tolist(), step["cu_seqlens"].tolist()
    held = [p for r in range(3) for p in table[r, :pu.pages_of(lens[r], P)].tolist()]
    free = [int(ring[(state[0] + i) % N]) for i in range(state[1])]
    assert sorted(held + free) == list(range(N))
    rows = slice(cu[2], cu[3])
    assert (step["slots"][rows] >= 0).all()
    x = pu.quarters(rng, (2, Hkv, 200, D))
    mala.mala_paged_write(x[0].bfloat16().cuda(), x[1].bfloat16().cuda(), step["slots"], cache)
    q = pu.quarters(rng, (Hq, D), 4)
    got = mala.paged_decode(q[None].bfloat16().cuda(), cache, table[2:3].contiguous(), i32([112]), 112, 0.125, 0.0)
    o, lse, _, _, _ = pu.decode_seq(q.numpy(), x[0, :, rows].numpy(), x[1, :, rows].numpy(),
                                    np.ones(112, bool), 0.125, 0.0, 128, 112)
    to, tl = pu.decode_bounds(112, 0.125 * 2 * float(q.abs().sum(1).max()), 2.0, False)
    assert np.abs(got["o"][0].double().cpu().numpy() - o).max() <= to
    assert np.abs(got["lse"][0].double().cpu().numpy() - lse).max() <= tl
