"""What the binding of the rotation says to arguments that its structs cannot hold (CPU and GPU)."""
import numpy as np
import pytest
import torch

import paper_2609_32712_amd as mala

BAD = [(TypeError, dict(layout=1.0)), (TypeError, dict(layout="half")), (TypeError, dict(layout=None)),
       (ValueError, dict(layout=1 << 31)), (ValueError, dict(layout=-(1 << 31) - 1)), (TypeError, dict(scale="1")),
       (TypeError, dict(scale=None)), (TypeError, dict(scale=[1.0])), (TypeError, dict(scale=1j)),
       (ValueError, dict(scale=10 ** 400))]


@pytest.mark.parametrize("err,kw", BAD)
def test_turns(err, kw):
    f = torch.ones(32, dtype=torch.float64)
    a = dict(layout=0, scale=1.0)
    a.update(kw)
    with pytest.raises(err, match=list(kw)[0]):
        mala._rope_turn(None, f, a["layout"], a["scale"], 1, 3, -1)


def test_turns_that_fit():
    f = torch.ones(32, dtype=torch.float64)
    want = mala._rope_turn(None, f, 1, 0.5, 1, 3, -1)
    for layout, scale in ((True, 0.5), (np.int64(1), np.float32(0.5)), (mala.ROPE_INTERLEAVED, torch.tensor(0.5))):
        assert mala._rope_turn(None, f, layout, scale, 1, 3, -1) == want
    assert mala._rope_turn(None, f, 0, 2, 1, 3, -1) == mala._rope_turn(None, f, 0, 2.0, 1, 3, -1)


@pytest.mark.gpu
@pytest.mark.parametrize("err,kw", BAD)
def test_calls(err, kw):
    f, _ = mala.rope_frequencies(64, device="cuda")
    q = torch.ones((2, 3, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: mala.rope(q, None, None, f, **kw), lambda: mala.rope_bwd(q, None, None, f, **kw),
                 lambda: mala.mala_rope(q, None, q, None, None, f, **kw)):
        with pytest.raises(err):
            call()
    with pytest.raises(mala.MalaError, match="finite"):         # (an infinity as an fp32)
        mala.mala_rope(q, None, q, None, None, f, scale=1e39)
    assert (q == 1).all()
    many = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda").expand(1 << 31, 1, 64)
    with pytest.raises(ValueError, match="32 bits"):
        mala.mala_rope(many, None, many, None, None, f)


@pytest.mark.gpu
def test_more_tokens_than_32_bits_hold_are_refused():
    # (the low 32 bits of their number were passed on: 2^32 + 3 tokens wrote three)
    import block_util as bu
    T = (1 << 32) + 3
    if torch.cuda.mem_get_info()[0] < 5 * T:
        pytest.skip("needs 20 GB of GPU memory")
    f, _ = mala.rope_frequencies(64, device="cuda")
    cache, k, v, ks, vs = bu.block_cache(mala, 2, 1, 16, 64)
    x = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda").expand(1, T, 64)
    slots = torch.empty(T, dtype=torch.int32, device="cuda")
    slots[:3] = torch.arange(3)
    with pytest.raises(ValueError, match="32 bits"):
        mala.mala_paged_write(x, x, slots, cache)
    with pytest.raises(ValueError, match="32 bits"):
        mala.mala_paged_rope_write(None, None, x, x, None, slots, cache, f)
    one = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="32 bits"):
        mala.mala_paged_update(one(1), one(1), one((1, 4)), one(4), one(2), one(1), one(2), slots, slots, one(4), 16, 4)
    assert not k.view(torch.uint8).any() and not ks.view(torch.uint8).any()
