"""The paged decode's code does not depend on the compiler's contraction of products and sums
(CPU: compiles to gfx950 assembly, runs nothing).

Its two kernels at tau > 0 promise the same retained sets, and each batch size has one of
them: they must not owe that to the compiler's choice of fused operations.
"""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2609_32712_amd import build as libbuild
from test_contraction import _kernels

pytestmark = pytest.mark.skipif(not os.path.exists(libbuild.HIPCC), reason="needs hipcc")


def test_paged_decode_does_not_depend_on_contraction(tmp_path):
    src = os.path.join(libbuild.CSRC, "mala_paged_decode.hip")
    with ThreadPoolExecutor(2) as ex:
        std, off = ex.map(lambda a: _kernels(src, *a), (
            ([], str(tmp_path / "std.s")), (["-ffp-contract=off"], str(tmp_path / "off.s"))))
    assert any("paged_decode" in k for k in std) and any("paged_join" in k for k in std)
    assert std.keys() == off.keys()
    for k in std:
        assert len(std[k]) > 50, k
        assert std[k] == off[k], k
