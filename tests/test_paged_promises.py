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
