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
