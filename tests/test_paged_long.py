"""Paged decodes whose wavefronts work on long runs, and large ragged batches of them, on the GPU:
sampled heads against the 64-bit form.  Which branches the calls reach is tested on the CPU
(test_paged_order.py)."""
import random

import numpy as np
import pytest
import torch

import paper_2609_32712_amd as mala
import paged_util as pu

pytestmark = pytest.mark.gpu

DENSE, CHAIN, TEAM = 0, 1, 2


def _log_lens(seed, B, n, more):
    rng = random.Random(seed)
    return [int(2 ** rng.uniform(0, n.bit_length() - 1)) for _ in range(B - len(more))] + more


def _call(lens, Hq, Hkv, D, e4m3, tau, split, mode, dealt, long, cut, P=16):
    return dict(lens=lens, Hq=Hq, Hkv=Hkv, D=D, e4m3=e4m3, tau=tau, split=split, mode=mode,
                dealt=dealt, long=long, cut=cut, P=P)


FEW = [30000, 20011, 12000, 700, 0, 33]
CALLS = dict(
    # runs of more than 32 tiles per wavefront (kTeam: per block), several blocks per sequence
    dense=_call(FEW, 64, 64, 64, False, 0.0, 256, DENSE, 1, True, 2),
    dense_e4m3=_call([60000, 41003, 777, 1], 32, 32, 128, True, 0.0, 256, DENSE, 1, True, 2, P=48),
    chain=_call([12000, 9000, 4097, 700, 0, 33], 64, 64, 64, False, 3.0, 4096, CHAIN, 1, True, 1),
    chain_e4m3=_call([12000, 9000, 4097, 700], 96, 48, 128, True, 3.0, 2048, CHAIN, 1, True, 1, P=32),
    team=_call([9000, 5000], 8, 2, 128, False, 3.0, 2048, TEAM, 0, True, 3),
    team_d64=_call([20000, 4096, 10], 8, 1, 64, False, 3.0, 4096, TEAM, 0, True, 2, P=64),
    # the same where many tiles of a split are left out
    chain_few=_call([12000, 9000, 4097, 700, 0, 33], 64, 64, 64, False, 60.0, 4096, CHAIN, 1, True, 1),
    team_few=_call([9000, 5000], 8, 2, 128, False, 60.0, 2048, TEAM, 0, True, 3),
    # more than 64 sequences, dealt by the classes of their runs, several blocks per sequence
    ragged=_call(_log_lens(1, 130, 8192, [20000, 9000, 16000, 0]), 32, 8, 64, False, 0.0, 256,
                 DENSE, 1, False, 4),
    ragged_e4m3=_call(_log_lens(2, 90, 4096, [30000, 0, 12345]), 32, 4, 128, True, 0.0, 256, DENSE,
                      1, False, 4, P=80),
    ragged_rule=_call(_log_lens(3, 150, 2048, [9000, 8191, 0]), 32, 16, 128, False, 3.0, 256, CHAIN,
                      1, False, 2),
    # a batch of more than a thousand
    many=_call(_log_lens(4, 1100, 512, [6000, 5000]), 16, 16, 64, False, 0.0, 256, DENSE, 1, False, 2),
)


@pytest.mark.parametrize("name", CALLS)
def test_long_calls(name):
    c = CALLS[name]
    lens, Hq, Hkv, D, P, tau, split = (c[x] for x in ("lens", "Hq", "Hkv", "D", "P", "tau", "split"))
    rng, pages, B = np.random.default_rng(len(lens)), 300, len(lens)
    dtype = torch.float8_e4m3fn if c["e4m3"] else torch.bfloat16
    # one pool of values that are exact in both types; sequences are random pages of it
    kv = pu.quarters(rng, (2, pages, Hkv, P, D)).float()
    k, v = (x.to(dtype).cuda() for x in kv)
    q = pu.quarters(rng, (B, Hq, D), 8)
    table = rng.integers(0, pages, (B, pu.pages_of(max(lens), P))).astype(np.int32)
    scale = float(np.float32(D ** -0.5))
    got = mala.paged_decode(q.to(torch.bfloat16).cuda(), mala.PagedCache(k, v),
                            torch.from_numpy(table).cuda(),
                            torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), scale,
                            tau, split)
    tiles = got["head_tiles"].cpu().numpy()
    legal = np.array([-(-n // 32) for n in lens])
    assert got["counters"][mala.CNT_LEGAL] == legal.sum() * Hq
    assert got["counters"][mala.CNT_RETAINED] == tiles.sum()
    if tau == 0:
        assert (tiles == legal[:, None]).all()
    else:
        assert (tiles <= legal[:, None]).all() and tiles.sum() < legal.sum() * Hq
    o, lse = got["o"].double().cpu().numpy(), got["lse"].double().cpu().numpy()
    smax = scale * 2 * float(q.abs().sum(2).max())
    # a decision can differ where the test value lies within its rounding of tau: that of a split's
    # normaliser and of the scores (as in the rule's other tests)
    band = (split + 100) * pu.U24 + 16 * pu.U24 * (smax + 1)
    heads = sorted({0, Hq // 2 + 1, Hq - 1})
    sampled = list(range(B)) if B < 200 else list(range(0, B, 8)) + list(range(B - 4, B))
    clear = 0
    for b in sampled:
        n = lens[b]
        if n == 0:
            assert (o[b] == 0).all() and np.isneginf(lse[b]).all()
            continue
        pos = np.arange(n)
        for h in heads:
            rows = kv[:, table[b, pos // P], h // (Hq // Hkv), pos % P].double().numpy()
            wo, wl, wt, _, tie = pu.decode_seq(q[b, h:h + 1].numpy(), rows[:1], rows[1:],
                                               np.ones(n, bool), scale, tau, split, n)
            if tie[0] <= band:
                continue
            clear += 1
            to, tl = pu.decode_bounds(n, smax, 2.0, False)
            assert tiles[b, h] == wt[0], (b, h)
            assert np.abs(o[b, h] - wo[0]).max() <= to, (b, h, np.abs(o[b, h] - wo[0]).max(), to)
            assert abs(lse[b, h] - wl[0]) <= tl, (b, h)
    assert clear >= 0.5 * len(heads) * sum(lens[b] > 0 for b in sampled)
