"""The paged KV cache without a GPU: refusals (all before any HIP call), workspace sizes, the
binding's argument checks, and the plain forms that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_32712_amd as mala
import paged_util as pu

BAD, UNSUP, WS = mala.MALA_ERR_INVALID_ARG, mala.MALA_ERR_UNSUPPORTED, mala.MALA_ERR_WORKSPACE


def _cache(**kw):
    a = dict(k_pages=256, v_pages=512, k_scale=None, v_scale=None, page_stride=4 * 32 * 128,
             head_stride=32 * 128, token_stride=128, num_pages=10, page_size=32, Hkv=4, D=128,
             dtype=mala.CACHE_BF16)
    a.update(kw)
    return mala._PagedCacheStruct(**a)


def _refused(status, want):
    assert status == want
    assert mala.load_library().mala_last_error().decode() != ""


CACHE_REFUSALS = [
    (dict(k_pages=None), BAD), (dict(v_pages=None), BAD), (dict(num_pages=0), BAD),
    (dict(page_size=0), BAD), (dict(page_size=-16), BAD), (dict(Hkv=0), BAD), (dict(dtype=2), BAD),
    (dict(k_scale=64), BAD), (dict(D=96), UNSUP), (dict(page_size=24), UNSUP),
    (dict(page_size=8), UNSUP), (dict(num_pages=1 << 27), UNSUP), (dict(token_stride=64), BAD),
    (dict(token_stride=132), BAD), (dict(head_stride=0), BAD), (dict(page_stride=-4096), BAD),
    (dict(token_stride=1 << 27), UNSUP), (dict(page_stride=1 << 60), UNSUP),
    (dict(k_pages=264), BAD), (dict(dtype=mala.CACHE_E4M3, token_stride=136), BAD),
]


@pytest.mark.parametrize("kw,want", CACHE_REFUSALS)
def test_every_entry_point_refuses_a_bad_cache(kw, want):
    lib = mala.load_library()
    c = ctypes.byref(_cache(**kw))
    _refused(lib.mala_paged_write(16, 16, 512, 128, 16, c, 4, None), want)
    _refused(lib.mala_paged_write(16, 16, 512, 128, 16, c, 0, None), want)
    _refused(lib.mala_paged_read(c, 16, 16, 16, 16, 2, 4, 100, 200, None), want)
    _refused(lib.mala_paged_decode(16, c, 16, 16, 16, 16, None, None, 64, 16, 1 << 30, 2, 8, 4,
                                   128, 0.1, 0.0, 0, None), want)


def test_null_cache():
    lib = mala.load_library()
    _refused(lib.mala_paged_write(16, 16, 512, 128, 16, None, 4, None), BAD)
    _refused(lib.mala_paged_read(None, 16, 16, 16, 16, 2, 4, 100, 200, None), BAD)


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(slots=None), BAD), (dict(T=-1), BAD),
    (dict(k=24), BAD), (dict(ts=516), BAD), (dict(hs=-128), BAD), (dict(ts=1 << 62), UNSUP)])
def test_write_refusals(kw, want):
    a = dict(k=16, v=32, ts=512, hs=128, slots=16, T=4)
    a.update(kw)
    _refused(mala.load_library().mala_paged_write(a["k"], a["v"], a["ts"], a["hs"], a["slots"],
                                                  ctypes.byref(_cache()), a["T"], None), want)


def test_write_of_no_tokens_is_done_at_once():
    assert mala.load_library().mala_paged_write(None, None, 0, 0, None, ctypes.byref(_cache()), 0,
                                                None) == mala.MALA_OK


@pytest.mark.parametrize("kw,want", [
    (dict(table=None), BAD), (dict(cu=None), BAD), (dict(k=None), BAD), (dict(S=0), BAD),
    (dict(W=0), BAD), (dict(mx=0), BAD), (dict(total=0), BAD), (dict(mx=129), BAD),
    (dict(v=40), BAD), (dict(total=1 << 24), UNSUP)])
def test_read_refusals(kw, want):
    a = dict(table=16, cu=16, k=16, v=32, S=2, W=4, mx=128, total=200)
    a.update(kw)
    _refused(mala.load_library().mala_paged_read(ctypes.byref(_cache()), a["table"], a["cu"],
                                                 a["k"], a["v"], a["S"], a["W"], a["mx"],
                                                 a["total"], None), want)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), BAD), (dict(table=None), BAD), (dict(lens=None), BAD), (dict(o=None), BAD),
    (dict(lse=None), BAD), (dict(split=0), BAD), (dict(split=48), BAD), (dict(split=-32), BAD),
    (dict(B=0), BAD), (dict(Hq=6), BAD), (dict(W=0), BAD), (dict(mx=0), BAD), (dict(mx=129), BAD),
    (dict(scale=0.0), BAD), (dict(scale=float("nan")), BAD), (dict(tau=-1.0), BAD),
    (dict(tau=float("inf")), BAD), (dict(tau=float("nan")), BAD), (dict(out=2), BAD),
    (dict(q=24), BAD), (dict(o=20), BAD), (dict(W=4000, mx=128000, ws=None), WS),
    (dict(W=4000, mx=128000, nbytes=100), WS), (dict(W=4000, mx=128000, ws=24), WS),
    (dict(B=1 << 28), UNSUP), (dict(B=1 << 21, mx=32), UNSUP),
    (dict(W=1 << 27, mx=2 ** 31 - 1), UNSUP), (dict(W=1 << 26, mx=1 << 30, B=1 << 6), UNSUP)])
def test_decode_refusals(kw, want):
    a = dict(q=16, table=16, lens=16, o=16, lse=16, split=64, ws=32, nbytes=1 << 62, B=2, Hq=8,
             W=4, mx=128, scale=0.1, tau=1e-3, out=0)
    a.update(kw)
    _refused(mala.load_library().mala_paged_decode(
        a["q"], ctypes.byref(_cache()), a["table"], a["lens"], a["o"], a["lse"], None, None,
        a["split"], a["ws"], a["nbytes"], a["B"], a["Hq"], a["W"], a["mx"], a["scale"], a["tau"],
        a["out"], None), want)


NAMES = ("lens", "new_lens", "table", "ring", "state", "lens_out", "cu", "slots", "positions",
         "state_out")


@pytest.mark.parametrize("kw,want", [(dict([(n, None)]), BAD) for n in NAMES if n != "positions"] + [
    (dict(R=0), BAD), (dict(W=0), BAD), (dict(P=0), BAD), (dict(num_pages=0), BAD),
    (dict(C=0), BAD), (dict(T=-1), BAD), (dict(P=20), UNSUP), (dict(R=1 << 20, W=1 << 10), UNSUP),
    (dict(num_pages=1 << 28), UNSUP), (dict(lens_out=0), BAD), (dict(state_out=4), BAD),
    (dict(slots=2), BAD), (dict(positions=7), BAD), (dict(ring=2), BAD)])
def test_update_refusals(kw, want):
    a = {n: 16 * (i + 1) for i, n in enumerate(NAMES)}
    a.update(R=4, W=8, P=16, num_pages=100, C=100, T=64)
    for n, x in kw.items():     # an index: the argument that it would share its memory with
        a[n] = a[NAMES[x]] if n in NAMES and x is not None else x
    _refused(mala.load_library().mala_paged_update(
        *(a[n] for n in NAMES), a["R"], a["W"], a["P"], a["num_pages"], a["C"], a["T"], None), want)


def test_workspace_size():
    f = mala.mala_paged_decode_workspace_size
    assert f(4, 32, 8, 128, 131072, 512) >= 4 * 32 * 2 * 132 * 4
    for bad in ((0, 32, 8, 128, 100, 64), (4, 32, 7, 128, 100, 64), (4, 32, 8, 96, 100, 64),
                (4, 32, 8, 128, 0, 64), (4, 32, 8, 128, 100, 48), (4, 32, 8, 128, 100, 0)):
        assert f(*bad) == 0
    assert f(1, 8, 2, 128, 1, 512) == 0          # one workgroup per head: no partials


def test_default_split_tokens():
    for B, H, n in ((1, 1, 1), (1, 8, 4096), (64, 8, 16384), (1, 1, 1 << 20)):
        s = mala.default_split_tokens(B, H, n)
        assert 64 <= s <= 512 and s % 32 == 0


def test_binding_refuses_cpu_tensors_and_wrong_types():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="CUDA"):
        mala.PagedCache(k, k.clone())
    with pytest.raises(TypeError, match="dtype"):
        mala.PagedCache(k.float(), k.float())
    with pytest.raises(TypeError, match="dtype"):
        mala.PagedCache(k, k.float())
    with pytest.raises(ValueError, match="4-d"):
        mala.PagedCache(k[0], k[0])
    with pytest.raises(ValueError, match="strides"):
        mala.PagedCache(k, torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16).transpose(1, 2))
    with pytest.raises(ValueError, match="contiguous"):
        t = torch.zeros((4, 2, 64, 16), dtype=torch.bfloat16).transpose(2, 3)
        mala.PagedCache(t, t)
    with pytest.raises(TypeError, match="PagedCache"):
        mala.mala_paged_write(k[0], k[0], torch.zeros(16, dtype=torch.int32), (k, k))
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="block_table"):
        mala.mala_paged_update(i, i, i, i, i, i, i, i, None, i, 16, 4)
    with pytest.raises(ValueError, match="two entries"):
        mala.mala_paged_update(i, i, torch.zeros((4, 2), dtype=torch.int32), i, i[:1], i,
                               torch.zeros(5, dtype=torch.int32), i, None, i, 16, 4)
    with pytest.raises(TypeError, match="CUDA"):
        mala.paged_update(i, i, torch.zeros((4, 2), dtype=torch.int32), i, i, 8, 16, 4)


# ------------------------------------------------------------------ the plain forms themselves
def test_plain_decode_is_softmax_attention_and_the_oracles_rule():
    rng = np.random.default_rng(0)
    n, D, Hq, Hkv = 256, 64, 4, 2
    q, k, v = rng.standard_normal((Hq, D)), rng.standard_normal((Hkv, n, D)), rng.standard_normal((Hkv, n, D))
    q[0] += 4 * k[0, 100]
    q[3] += 3 * k[1, 250]
    seen = np.ones(n, dtype=bool)
    o, lse, tiles, _, _ = pu.decode_seq(q, k, v, seen, 0.125, 0.0, 64, n)
    s = np.einsum("hd,hnd->hn", q, k.repeat(2, 0)) * 0.125
    p = np.exp(s - s.max(1, keepdims=True))
    np.testing.assert_allclose(o, np.einsum("hn,hnd->hd", p / p.sum(1, keepdims=True), v.repeat(2, 0)), atol=1e-12)
    np.testing.assert_allclose(lse, np.log(np.exp(s).sum(1)), atol=1e-12)
    assert (tiles == 8).all()
    for tau in (0.3, 1.0):
        o, lse, tiles, keep, _ = pu.decode_seq(q, k, v, seen, 0.125, tau, 64, n)
        ref = pu.oracle_decode(q, k, v, 0.125, tau, n // 64)
        np.testing.assert_array_equal(tiles, ref["tiles"][0])
        np.testing.assert_allclose(o, ref["o"][0], atol=1e-12)
        np.testing.assert_allclose(lse, ref["lse"][0], atol=1e-12)
        assert tiles.min() < 8


def test_plain_update_keeps_every_page_once():
    rng = np.random.default_rng(1)
    P, R, W, N = 16, 12, 6, 50
    table, ring = np.full((R, W), -1, np.int32), rng.permutation(N).astype(np.int32)
    lens, state = np.zeros(R, np.int32), np.array([0, N], np.int32)
    for step in range(60):
        new = np.where(rng.random(R) < 0.25, 0, lens + rng.integers(-20, 40, R)).astype(np.int32)
        before = lens.copy()
        lens, cu, slots, pos, out = pu.update_plain(lens, new, table, ring, state, P, N, 600)
        state = out[:2]
        used = [table[r, j] for r in range(R) for j in range(pu.pages_of(lens[r], P))]
        free = [ring[(state[0] + i) % N] for i in range(state[1])]
        assert sorted(used + free) == list(range(N))
        for r in range(R):
            for t in range(cu[r], cu[r + 1]):
                want = table[r, pos[t] // P] * P + pos[t] % P if lens[r] > before[r] else -1
                assert slots[t] == want
