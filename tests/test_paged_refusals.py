"""Refusals of the paged KV cache at the ends of the argument types (CPU: all come before any
HIP call)."""
import ctypes

import pytest

import paper_2609_32712_amd as mala
from test_paged_abi import BAD, UNSUP, _cache, _refused


@pytest.mark.parametrize("kw", [
    # products of a stride that pass 2^63: 16 rows of 2^59 bf16 elements are 2^64 bytes
    dict(num_pages=1, token_stride=1 << 59), dict(num_pages=1, token_stride=1 << 60),
    dict(num_pages=1, token_stride=(1 << 59) + 128), dict(num_pages=1, token_stride=(1 << 62) - 64),
    dict(num_pages=1, head_stride=1 << 61), dict(num_pages=1, Hkv=1 << 20, head_stride=1 << 43),
    dict(num_pages=1, Hkv=1, head_stride=(1 << 62) - 64),
    dict(num_pages=1, page_stride=(1 << 62) - 64), dict(num_pages=1 << 20, page_stride=1 << 42),
    dict(num_pages=1, dtype=mala.CACHE_E4M3, token_stride=1 << 60),
    dict(num_pages=1, dtype=mala.CACHE_E4M3, head_stride=1 << 62)])
def test_cache_strides_whose_products_pass_64_bits(kw):
    lib, c = mala.load_library(), ctypes.byref(_cache(**kw))
    _refused(lib.mala_paged_write(16, 16, 512, 128, 16, c, 0, None), UNSUP)
    _refused(lib.mala_paged_read(c, 16, 16, 16, 16, 2, 4, 100, 0, None), UNSUP)
    _refused(lib.mala_paged_decode(16, c, 16, 16, 16, 16, None, None, 64, 16, 1 << 30, 2, 6, 4,
                                   128, 0.1, -1.0, 0, None), UNSUP)


@pytest.mark.parametrize("kw", [dict(num_pages=1, head_stride=1 << 40), dict(token_stride=(1 << 26) - 64),
                                dict(num_pages=1 << 20, page_stride=1 << 38)])
def test_large_cache_strides_that_fit(kw):
    assert mala.load_library().mala_paged_write(16, 16, 512, 128, 16, ctypes.byref(_cache(**kw)), 0,
                                                None) == mala.MALA_OK


# name, entries of each of mala_paged_update's arrays for R = 4, W = 8, C = 100, T = 64
UPDATE = (("lens", 4), ("new_lens", 4), ("table", 32), ("ring", 100), ("state", 2), ("lens_out", 4),
          ("cu", 5), ("slots", 64), ("positions", 64), ("state_out", 4))


def _update(at, T=64):
    return mala.load_library().mala_paged_update(*(at[n] for n, _ in UPDATE), 4, 8, 16, 100, 100, T, None)


def _apart():
    at, out = 4096, {}
    for name, n in UPDATE:
        out[name] = at
        at += 4 * n                       # one behind the other, without a gap
    return out


OUTPUTS = [n for n, _ in UPDATE[5:]]
PAIRS = [(o, n) for o in OUTPUTS for n, _ in UPDATE if n != o] + [("ring", "table")]


@pytest.mark.parametrize("out,other", PAIRS)
def test_update_refuses_arrays_that_overlap(out, other):
    size = dict(UPDATE)
    for shift in (-4 * (size[out] - 1), 0, 4 * (size[other] - 1)):     # by one entry, from either end
        at = {n: (1 << 20) + (i << 12) for i, (n, _) in enumerate(UPDATE)}
        at[out] = at[other] + shift
        _refused(_update(at), BAD)


def test_update_takes_arrays_that_touch():
    # (a status of its own: without a GPU the launch fails, behind all refusals)
    import torch
    if torch.cuda.is_available():
        pytest.skip("addresses of no tensors: for machines without a GPU")
    assert _update(_apart()) == mala.MALA_ERR_HIP
    # arrays of no entries overlap nothing, wherever they are
    at = _apart()
    at["slots"] = at["positions"] = at["table"] + 8
    assert _update(at, T=0) == mala.MALA_ERR_HIP


def test_default_split_does_not_go_by_the_batch(monkeypatch):
    import torch
    seen = []
    monkeypatch.setattr(mala, "mala_paged_decode", lambda *a, **kw: seen.append(a[9]))

    class Cache:
        Hkv = 4
    for B, n in ((1, 100), (1, 100000), (64, 100), (200, 30000)):
        mala.paged_decode(torch.zeros((B, 8, 64)), Cache, None, None, n, 0.125, 1e-3)
        mala.paged_decode(torch.zeros((B, 8, 64)), Cache, None, None, n, 0.125, 1e-3, 512)
    assert seen[1::2] == [512] * 4 and set(seen[::2]) == {mala.default_split_tokens()}


def _handle():
    """A cache handle without tensors (the constructor takes those of a GPU only)."""
    c = object.__new__(mala.PagedCache)
    object.__setattr__(c, "_struct", _cache())
    object.__setattr__(c, "_ref", ctypes.byref(c._struct))
    for n in ("k_pages", "v_pages", "k_scale", "v_scale", "Hkv", "D", "device", "num_pages", "page_size"):
        object.__setattr__(c, n, getattr(c._struct, n, -1))
    return c


@pytest.mark.parametrize("name", ["k_pages", "v_pages", "k_scale", "v_scale", "Hkv", "D", "num_pages",
                                  "page_size", "device", "_ref"])
def test_a_cache_handle_does_not_change(name):
    # its addresses were taken when it was made: other tensors would be kept but not used, and the
    # first ones used but not kept
    c = _handle()
    with pytest.raises(AttributeError, match="PagedCache"):
        setattr(c, name, 1)
    with pytest.raises(AttributeError, match="PagedCache"):
        delattr(c, name)
    c.note = 1                            # (a caller's own)
    del c.note


@pytest.mark.parametrize("big", [1 << 31, (1 << 32) + 64, -(1 << 31) - 1, 1 << 70])
def test_the_binding_refuses_numbers_that_do_not_fit(monkeypatch, big):
    # ctypes would pass their low 32 bits on: 2^32 + 64 as 64
    import torch
    monkeypatch.setattr(mala, "_args", lambda *a: None)
    monkeypatch.setattr(mala, "_device", lambda *a: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    called = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: called.append((name, a)) or 0
    monkeypatch.setattr(mala, "_lib", Lib())
    c, i = _handle(), torch.zeros(4, dtype=torch.int32)
    table, q, kv = torch.zeros((4, 4), dtype=torch.int32), torch.zeros((4, 8, 128)), torch.zeros((4, 9, 128))
    read = lambda n: mala.mala_paged_read(c, table, i, n, kv, kv)
    decode = lambda n, split: mala.mala_paged_decode(q, c, table, i, n, q, q, None, None, split, None, 0.1, 0.0)
    update = lambda page, pages: mala.mala_paged_update(i, i, table, i, i, i, i, i, None, i, page, pages)
    for call, good in ((read, (64,)), (decode, (64, 128)), (update, (16, 100))):
        call(*good)
        assert len(called) == 1 and all(n in called[0][1] for n in good)
        called.clear()
        for j in range(len(good)):
            with pytest.raises((ValueError, OverflowError), match="32 bits"):
                call(*good[:j], big, *good[j + 1:])
        assert not called
    with pytest.raises((ValueError, OverflowError), match="32 bits"):
        mala.mala_paged_decode_workspace_size(4, 8, 2, 128, big, 64)


@pytest.mark.parametrize("kw", [dict(T=1 << 28), dict(T=1 << 29, dtype=mala.CACHE_E4M3),
                                dict(T=(1 << 31) - 1, D=64, token_stride=64)])
def test_write_refuses_a_launch_of_2_to_the_32_threads(kw):
    T = kw.pop("T")
    c = ctypes.byref(_cache(**kw))
    _refused(mala.load_library().mala_paged_write(16, 32, 512, 128, 16, c, T, None), UNSUP)
