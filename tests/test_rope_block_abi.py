"""Rotary positions and the cache with a scale per block without a GPU: refusals (all before any
HIP call), the binding's checks, the frequencies, and the plain forms the GPU tests compare with."""
import ctypes
import math

import numpy as np
import pytest
import torch

import block_util as bu
import paged_util as pu
import paper_2609_32712_amd as mala

BAD, UNSUP = mala.MALA_ERR_INVALID_ARG, mala.MALA_ERR_UNSUPPORTED


def _refused(status, want):
    assert status == want, mala.load_library().mala_last_error()
    assert mala.load_library().mala_last_error().decode() != ""


def _rows(**kw):
    a = dict(x=1 << 20, out=1 << 30, xb=4096, xh=128, xt=1024, ob=4096, oh=128, ot=1024, heads=4)
    a.update(kw)
    return mala._ROPE_ROWS.pack(*a.values())


def _turn(**kw):
    a = dict(pos=64, stride=0, freq=64, R=128, layout=0, scale=1.0)
    a.update(kw)
    return mala._ROPE.pack(*a.values())


def _rope(q=None, k=None, turn=None, B=2, T=4, D=128, i=1, o=1, inverse=0):
    return mala.load_library().mala_rope(q or _rows(), k, turn or _turn(), B, T, D, i, o, inverse, None)


ROW_REFUSALS = [
    (dict(x=0), BAD), (dict(out=0), BAD), (dict(heads=0), BAD), (dict(heads=-1), BAD),
    (dict(heads=65536), UNSUP), (dict(x=(1 << 20) + 8), BAD), (dict(out=(1 << 30) + 4), BAD),
    (dict(xt=-1024), BAD), (dict(xh=132), BAD), (dict(ot=1028), BAD), (dict(oh=64), BAD),
    (dict(ot=0), BAD), (dict(xt=1 << 60), UNSUP), (dict(ob=1 << 60), UNSUP),
    # outputs that meet their input without being it: a part of it, shifted, other strides
    (dict(out=(1 << 20) + 256), BAD), (dict(out=1 << 20, ot=2048, ob=8192), BAD),
    (dict(out=(1 << 20) - 16), BAD)]
TURN_REFUSALS = [
    (dict(freq=0), BAD), (dict(R=0), BAD), (dict(R=-16), BAD), (dict(R=144), BAD), (dict(R=24), UNSUP),
    (dict(R=8), UNSUP), (dict(layout=2), BAD), (dict(layout=-1), BAD), (dict(scale=math.inf), BAD),
    (dict(scale=math.nan), BAD), (dict(freq=68), BAD), (dict(pos=66), BAD), (dict(stride=-1), BAD),
    (dict(stride=1 << 62), UNSUP)]


@pytest.mark.parametrize("kw,want", ROW_REFUSALS)
def test_rows_are_refused(kw, want):
    _refused(_rope(q=_rows(**kw)), want)
    _refused(_rope(k=_rows(**kw)), want)
    kw = {n: x for n, x in kw.items() if n not in ("xb", "ob")}
    if kw:
        c = ctypes.byref(_block_cache())
        _refused(mala.load_library().mala_paged_rope_write(_rows(**kw), 256, 512, 512, 128, 16, _turn(), c, 8,
                                                           None), want)


@pytest.mark.parametrize("kw,want", TURN_REFUSALS)
def test_turns_are_refused(kw, want):
    _refused(_rope(turn=_turn(**kw)), want)
    _refused(_rope(turn=_turn(**kw), T=0), want)
    if "stride" not in kw or kw["stride"] < 0:
        c = ctypes.byref(_block_cache())
        _refused(mala.load_library().mala_paged_rope_write(None, 256, 512, 512, 128, 16, _turn(**kw), c, 4,
                                                           None), want)


@pytest.mark.parametrize("kw,want", [
    (dict(B=-1), BAD), (dict(T=-1), BAD), (dict(D=96), UNSUP), (dict(D=256), UNSUP), (dict(i=2), BAD),
    (dict(o=-1), BAD), (dict(B=1 << 16, T=1 << 16), UNSUP)])
def test_rope_sizes_are_refused(kw, want):
    _refused(_rope(**kw), want)


def test_rope_nulls_and_nothing_to_do():
    lib = mala.load_library()
    _refused(lib.mala_rope(None, None, _turn(), 1, 1, 128, 1, 1, 0, None), BAD)
    _refused(lib.mala_rope(_rows(), None, None, 1, 1, 128, 1, 1, 0, None), BAD)
    for kw in (dict(B=0), dict(T=0), dict(B=0, T=0)):
        assert _rope(**kw) == mala.MALA_OK
        assert _rope(q=_rows(x=0, out=0), **kw) == mala.MALA_OK


def _block_cache(**kw):
    a = dict(k_pages=256, v_pages=512, k_scale=None, v_scale=None, page_stride=4 * 32 * 128,
             head_stride=32 * 128, token_stride=128, num_pages=10, page_size=32, Hkv=4, D=128,
             dtype=mala.CACHE_E4M3_BLOCK, k_block_scale=64, v_block_scale=1 << 16)
    a.update(kw)
    return mala._PagedCacheStruct(**a)


@pytest.mark.parametrize("kw,want", [
    (dict(k_block_scale=None), BAD), (dict(v_block_scale=None), BAD), (dict(k_scale=64), BAD),
    (dict(v_scale=64), BAD), (dict(dtype=3), BAD), (dict(token_stride=136), BAD), (dict(D=96), UNSUP),
    (dict(page_size=24), UNSUP), (dict(k_pages=264), BAD), (dict(num_pages=1 << 27), UNSUP),
    (dict(v_block_scale=64), BAD), (dict(v_block_scale=64 + 79), BAD), (dict(k_block_scale=(1 << 16) + 79), BAD)])
def test_block_caches_are_refused(kw, want):
    lib, c = mala.load_library(), ctypes.byref(_block_cache(**kw))
    _refused(lib.mala_paged_write(256, 512, 512, 128, 16, c, 4, None), want)
    _refused(lib.mala_paged_read(c, 16, 16, 16, 16, 2, 4, 100, 200, None), want)
    _refused(lib.mala_paged_decode(16, c, 16, 16, 16, 16, None, None, 64, 16, 1 << 30, 2, 8, 4, 128, 0.1,
                                   0.0, 0, None), want)
    _refused(lib.mala_paged_rope_write(None, 256, 512, 512, 128, 16, _turn(), c, 4, None), want)


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(slots=None), BAD), (dict(T=-1), BAD), (dict(k=24), BAD),
    (dict(ts=516), BAD), (dict(hs=-128), BAD), (dict(ts=1 << 62), UNSUP), (dict(T=(1 << 31) - 1), UNSUP),
    (dict(turn=None), BAD), (dict(cache=None), BAD)])
def test_rope_write_refusals(kw, want):
    for dtype in range(3):
        a = dict(k=256, v=512, ts=512, hs=128, slots=16, turn=_turn(), T=4,
                 cache=ctypes.byref(_block_cache(dtype=dtype)))
        a.update(kw)
        lib = mala.load_library()
        call = lambda q, a=a: lib.mala_paged_rope_write(q, a["k"], a["v"], a["ts"], a["hs"], a["slots"],
                                                        a["turn"], a["cache"], a["T"], None)
        _refused(call(None), want)
        _refused(call(_rows()), want)
        if "turn" not in kw and "cache" not in kw:
            _refused(lib.mala_paged_write(a["k"], a["v"], a["ts"], a["hs"], a["slots"], a["cache"], a["T"],
                                          None), want)
    # no tokens: nothing else is looked at
    a = ctypes.byref(_block_cache())
    assert mala.load_library().mala_paged_rope_write(None, None, None, 0, 0, None, _turn(), a, 0, None) == 0


# ------------------------------------------------------------------ the binding (CPU tensors: refused too)
def test_binding_checks_rope():
    q, f = torch.zeros(4, 3, 128).bfloat16(), torch.ones(64, dtype=torch.float64)
    for bad in (lambda: mala.mala_rope(q, None, q, None, None, f),                    # not on the GPU
                lambda: mala.rope(q, None, None, f), lambda: mala.rope_bwd(q, None, None, f)):
        with pytest.raises(TypeError):
            bad()
    for shape in ((128,), (3, 128), (1, 1, 4, 3, 128)):
        with pytest.raises(ValueError):
            x = torch.zeros(shape).bfloat16()
            mala.mala_rope(x, None, x, None, None, f)
    with pytest.raises(ValueError):
        mala.mala_rope([1.0], None, q, None, None, f)


def test_binding_checks_block_caches():
    k = torch.zeros(6, 2, 32, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = lambda *shape: torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    good = s(6, 2, 2)
    with pytest.raises(TypeError):        # all right but for the device
        mala.PagedCache(k, k.clone(), good, good.clone())
    for ks, vs, err in ((good, None, TypeError), (None, good, TypeError), (good, torch.ones(2), TypeError),
                        (s(6, 2, 1), good, ValueError), (good, s(6, 2, 4)[..., ::2], ValueError),
                        (good.view(torch.uint8), good.view(torch.uint8), TypeError)):
        with pytest.raises(err):
            mala.PagedCache(k, k.clone(), ks, vs)
    with pytest.raises(TypeError):
        mala.PagedCache(torch.zeros(6, 2, 32, 64).bfloat16(), torch.zeros(6, 2, 32, 64).bfloat16(), good, good)


# ------------------------------------------------------------------ frequencies
def test_frequencies():
    f, s = mala.rope_frequencies(64, 10000.0)
    assert f.dtype == torch.float64 and f.shape == (32,) and s == 1.0
    np.testing.assert_allclose(f.numpy(), [10000.0 ** (-i / 32) for i in range(32)], rtol=1e-14)
    lin, s = mala.rope_frequencies(64, 10000.0, 4.0, "linear")
    np.testing.assert_allclose(lin.numpy(), f.numpy() / 4, rtol=1e-14)
    ntk, s = mala.rope_frequencies(64, 10000.0, 4.0, "ntk")
    assert s == 1.0 and ntk[0] == 1.0 and abs(ntk[-1] * 4 / f[-1] - 1) < 1e-12
    assert (ntk[1:] < f[1:]).all() and (ntk >= f / 4 * (1 - 1e-12)).all()
    yarn, s = mala.rope_frequencies(64, 10000.0, 4.0, "yarn", original_len=4096)
    turns = 4096 * f / (2 * math.pi)
    fast, slow = turns >= 32, turns <= 1
    assert fast.any() and slow.any() and (~fast & ~slow).any()
    assert torch.equal(yarn[fast], f[fast]) and torch.equal(yarn[slow], f[slow] / 4)
    between = ~fast & ~slow
    w = (turns[between] - 1) / 31
    np.testing.assert_allclose(yarn[between].numpy(), (w * f[between] + (1 - w) * f[between] / 4).numpy(),
                               rtol=1e-12)
    assert abs(s - (0.1 * math.log(4) + 1)) < 1e-15
    assert mala.rope_frequencies(64, factor=0.5, scaling="yarn", original_len=4096)[1] == 1.0
    for kw in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=64, base=-1.0),
               dict(rotary_dim=64, factor=0.0), dict(rotary_dim=64, factor=math.inf),
               dict(rotary_dim=64, scaling="other"), dict(rotary_dim=64, scaling="yarn"),
               dict(rotary_dim=2, scaling="ntk", factor=2.0),
               dict(rotary_dim=64, scaling="yarn", original_len=4096, beta_fast=1.0)):
        with pytest.raises(ValueError):
            mala.rope_frequencies(**kw)


# ------------------------------------------------------------------ the plain forms
def test_plain_e4m3_is_torchs():
    y = np.concatenate([np.linspace(-448, 448, 20001), np.ldexp(1.0 + np.arange(64) / 64, np.arange(-12, 52) % 20 - 12),
                        [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11]])
    want = torch.from_numpy(y).float().to(torch.float8_e4m3fn).float().double().numpy()
    got = bu.e4m3(y.astype(np.float32).astype(np.float64))
    assert (got == want).all()


def test_plain_exponents():
    assert bu.exponent(np.array([0.0, math.nan, math.inf])) == bu.E_MIN
    for e in (-117, -5, 0, 100, 119):
        assert bu.exponent(np.array([math.ldexp(448.0, e), 0.0])) == e
        assert bu.exponent(np.array([math.ldexp(450.0, e)])) == e + 1
    assert bu.exponent(np.array([float(torch.finfo(torch.bfloat16).max)])) == 120
    assert bu.exponent(np.array([2.0 ** -133])) == -117


def test_plain_rotation_keeps_lengths_and_its_inverse_undoes_it():
    rng = np.random.default_rng(1)
    x, f = rng.standard_normal((2, 5, 64)), mala.rope_frequencies(32)[0].numpy()
    pos = np.array([0, 1, -7, 100000, 2 ** 31 - 1])
    for layout in (0, 1):
        y = bu.turned(x, pos, f, layout, 1.0)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
        assert (y[:, 0] == x[:, 0]).all() and (y[..., 32:] == x[..., 32:]).all()
        np.testing.assert_allclose(bu.turned(y, pos, f, layout, 1.0, True), x, atol=1e-12)
    # scores go by the distance alone
    a, b = rng.standard_normal((2, 1, 64))
    d = [float((bu.turned(a, np.array([p + 3]), f, 0, 1.0) * bu.turned(b, np.array([p]), f, 0, 1.0)).sum())
         for p in (0, 50)]
    assert abs(d[0] - d[1]) < 1e-12


def test_plain_blocks():
    # a block of one token, then a larger one (the first is rounded again), then anew from row 0
    v, e = np.full((1, 1, 16, 4), 3.0), np.full((1, 1, 1), 99, np.int64)
    bu.write_plain(v, e, np.array([[[1.0, 0.5, 3.5, -7.0]]]), [0])
    assert e[0, 0, 0] == -6 and (v[0, 0, 0] == [64, 32, 224, -448]).all() and (v[0, 0, 1:] == 3).all()
    # (100 over 2^-2 is 400, between 384 and 416: to the even one)
    bu.write_plain(v, e, np.array([[[0.0, 0.0, 0.0, 100.0]]]), [5])
    assert e[0, 0, 0] == -2 and (v[0, 0, 0] == [4, 2, 14, -28]).all() and v[0, 0, 5, 3] == 384
    assert (v[0, 0, 1] == 0.1875).all()
    bu.write_plain(v, e, np.array([[[0.0, 0.0, 0.0, 1.0]]]), [3])
    assert e[0, 0, 0] == -2 and v[0, 0, 3, 3] == 4 and (v[0, 0, 0] == [4, 2, 14, -28]).all()
    bu.write_plain(v, e, np.array([[[0.0, 0.0, 0.0, 1.0]], ])[:, [0, 0]], [0, 15])
    assert e[0, 0, 0] == -8 and v[0, 0, 0, 3] == 256 and v[0, 0, 5, 3] == 384
