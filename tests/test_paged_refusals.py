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
