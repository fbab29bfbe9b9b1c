"""The rotation's and the block-scaled write's code does not depend on the compiler's contraction of
products and sums (CPU: compiles to gfx950 assembly, runs nothing).

A rotated write promises the bits of a rotation and a write: they must not owe that to the
compiler's choice of fused operations.
"""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2609_32712_amd import build as libbuild
from test_contraction import _kernels

pytestmark = pytest.mark.skipif(not os.path.exists(libbuild.HIPCC), reason="needs hipcc")


@pytest.mark.parametrize("name,part", [("mala_rope.hip", "mala_rope_kernel"),
                                       ("mala_paged_block.hip", "mala_paged_block_rope")])
def test_rotations_do_not_depend_on_contraction(name, part, tmp_path):
    src = os.path.join(libbuild.CSRC, name)
    with ThreadPoolExecutor(2) as ex:
        std, off = ex.map(lambda a: _kernels(src, *a), (
            ([], str(tmp_path / "std.s")), (["-ffp-contract=off"], str(tmp_path / "off.s"))))
    assert any(part in k for k in std) and std.keys() == off.keys()
    for k in std:
        assert len(std[k]) > 50, k
        assert std[k] == off[k], k
