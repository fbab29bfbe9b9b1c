"""Rotary positions on the GPU against the definition in 64 bits: layouts, parts of a head, types,
strides, positions, in place, gradients, streams and graphs, and with the attention behind them."""
import numpy as np
import pytest
import torch

import block_util as bu
import paged_util as pu
import paper_2609_32712_amd as mala

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rows(rng, B, H, T, D, dtype, order="heads"):
    """[B, H, T, D] rows: contiguous, slices of [B, T, H, D] rows, or of every other head of wider ones."""
    x = torch.from_numpy(rng.standard_normal((B, H, T, D))).to(dtype)
    if order == "heads":
        return x.cuda()
    if order == "tokens":
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    wide = torch.zeros((T, B, 2 * H, 2 * D), dtype=dtype, device="cuda")
    view = wide[:, :, ::2, D:].permute(1, 2, 0, 3)
    view.copy_(x.cuda())
    return view


def check(got, x, pos, f, layout, scale, inverse=False):
    x64 = x.double().cpu().numpy()
    p = np.broadcast_to(pos, (x.shape[0], x.shape[2]))[:, None]
    want = bu.turned(x64, p, f, layout, scale, inverse)
    bound = bu.turned_bound(x64, f, layout, scale, got.dtype == BF16, int(np.abs(pos).max()))
    assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()


CASES = [
    # B, Hq, Hkv, T, D, R, layout, in, out, x order, out order, scale
    (1, 1, 1, 1, 64, 64, 0, BF16, BF16, "heads", "heads", 1.0),
    (1, 8, 2, 1, 128, 128, 0, BF16, BF16, "tokens", "tokens", 1.0),
    (2, 3, 1, 33, 128, 64, 0, BF16, F32, "tokens", "heads", 1.25),
    (1, 5, 5, 257, 64, 16, 1, F32, BF16, "wide", "heads", 1.0),
    (3, 7, 1, 31, 64, 48, 0, F32, F32, "heads", "wide", -0.5),
    (1, 32, 8, 65, 128, 128, 1, BF16, BF16, "wide", "tokens", 1.0),
    (2, 16, 2, 100, 128, 96, 1, F32, F32, "tokens", "tokens", 0.0),
    (1, 40, 8, 1000, 128, 112, 0, BF16, BF16, "tokens", "heads", 2.0),
    (5, 2, 1, 4097, 64, 32, 1, BF16, F32, "heads", "heads", 1.0),
]


@pytest.mark.parametrize("B,Hq,Hkv,T,D,R,layout,tin,tout,xo,oo,scale", CASES)
def test_rope(B, Hq, Hkv, T, D, R, layout, tin, tout, xo, oo, scale):
    rng = np.random.default_rng(T + D)
    f, _ = mala.rope_frequencies(R, device="cuda")
    q, k = rows(rng, B, Hq, T, D, tin, xo), rows(rng, B, Hkv, T, D, tin, xo)
    fn = f.cpu().numpy()
    for pos in (None, rng.integers(-5000, 200000, T), rng.integers(0, 1 << 24, (B, T))):
        p = None if pos is None else torch.from_numpy(pos).int().cuda()
        at = np.arange(T) if pos is None else pos
        for inverse in (False, True):
            qo, ko = rows(rng, B, Hq, T, D, tout, oo), rows(rng, B, Hkv, T, D, tout, oo)
            mala.mala_rope(q, k, qo, ko, p, f, layout, scale, inverse)
            check(qo, q, at, fn, layout, scale, inverse)
            check(ko, k, at, fn, layout, scale, inverse)
            # alone the same bits; nothing around the rows is written
            one = rows(rng, B, Hq, T, D, tout, "wide")
            around = one.permute(2, 0, 1, 3)._base
            around[:, :, 1::2] = 3.0
            around[..., :D] = 5.0
            mala.mala_rope(q, None, one, None, p, f, layout, scale, inverse)
            assert torch.equal(one, qo)
            assert (around[:, :, 1::2, D:] == 3.0).all() and (around[..., :D] == 5.0).all()


@pytest.mark.parametrize("far", [1 << 20, 1 << 27, (1 << 31) - 1])
@pytest.mark.parametrize("layout", [0, 1])
def test_far_positions(far, layout):
    # fp32 results stay right to fp32 where an fp32 angle would have lost every bit
    rng = np.random.default_rng(layout)
    f, _ = mala.rope_frequencies(128, device="cuda")
    pos = np.concatenate([[far, -far, far - 1, 0, -1], rng.integers(far // 2, far, 59)])
    q = rows(rng, 1, 2, 64, 128, F32)
    out = mala.rope(q, None, torch.from_numpy(pos).int().cuda(), f, layout, out_dtype=F32)["q"]
    check(out, q, pos, f.cpu().numpy(), layout, 1.0)


def test_quarter_turns():
    # multiples of a quarter turn and their neighbours, where the quadrant changes
    q = torch.ones((1, 64, 64), device="cuda")
    f = torch.full((32,), np.pi / 2, dtype=torch.float64, device="cuda")
    f[16:] = torch.nextafter(f[16:], torch.full_like(f[16:], 10.0))
    f[24:] = torch.nextafter(f[16:24], torch.full_like(f[24:], -10.0)) * 0.5
    pos = np.arange(-32, 32)
    out = mala.rope(q, None, torch.from_numpy(pos).int().cuda(), f, 0, out_dtype=F32)["q"]
    check(out[None], q[None], pos, f.cpu().numpy(), 0, 1.0)


def test_every_head_count_and_token_count():
    # head slices and token groups that do not divide: every row once
    rng = np.random.default_rng(5)
    f, _ = mala.rope_frequencies(64, device="cuda")
    for D in (64, 128):
        for Hq, Hkv in ((1, 1), (3, 1), (13, 1), (64, 8), (2, 2)):
            for T in (1, 7, 31, 32, 33, 64, 65, 511):
                q, k = rows(rng, 1, Hq, T, D, BF16, "tokens"), rows(rng, 1, Hkv, T, D, BF16)
                out = mala.rope(q, k, None, f)
                check(out["q"], q, np.arange(T), f.cpu().numpy(), 0, 1.0)
                check(out["k"], k, np.arange(T), f.cpu().numpy(), 0, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_slices_of_one_projection(dtype):
    rng = np.random.default_rng(6)
    T, Hq, Hkv, D = 77, 6, 2, 128
    f, _ = mala.rope_frequencies(D, device="cuda")
    proj = torch.from_numpy(rng.standard_normal((T, Hq + 2 * Hkv, D))).to(dtype).cuda()
    before = proj.clone()
    q, k = proj[:, :Hq].transpose(0, 1), proj[:, Hq:Hq + Hkv].transpose(0, 1)
    want = mala.rope(q, k, None, f, out_dtype=dtype)
    mala.mala_rope(q, k, q, k, None, f)
    assert torch.equal(q, want["q"]) and torch.equal(k, want["k"])
    assert torch.equal(proj[:, Hq + Hkv:], before[:, Hq + Hkv:])
    # an output that meets its input otherwise is refused
    with pytest.raises(mala.MalaError):
        mala.mala_rope(q, None, proj[:, 1:Hq + 1].transpose(0, 1), None, None, f)


def test_broadcast_input_and_no_tokens():
    rng = np.random.default_rng(7)
    f, _ = mala.rope_frequencies(64, device="cuda")
    one = rows(rng, 1, 1, 1, 64, BF16)
    x = one.expand(2, 3, 50, 64)               # one row for every position and head
    check(mala.rope(x, None, None, f)["q"], x, np.arange(50), f.cpu().numpy(), 0, 1.0)
    for shape in ((0, 3, 5, 64), (2, 3, 0, 64)):
        e = torch.empty(shape, dtype=BF16, device="cuda")
        assert mala.rope(e, e, None, f)["k"].shape == shape
        for pos in (shape[2:3], (shape[0], shape[2])):
            pos = torch.zeros(pos, dtype=torch.int32, device="cuda")
            assert mala.rope(e, None, pos, f)["q"].shape == shape


def test_infinities_and_nan_stay_in_their_pairs():
    f, _ = mala.rope_frequencies(32, device="cuda")
    q = torch.ones((1, 4, 64), device="cuda")
    q[0, 1, 3], q[0, 2, 40] = float("nan"), float("inf")
    out = mala.rope(q, None, None, f, out_dtype=F32)["q"][0]
    bad = torch.zeros((4, 64), dtype=torch.bool, device="cuda")
    bad[1, 3] = bad[1, 19] = bad[2, 40] = True
    assert (~out.isfinite() == bad).all() and out[2, 40] == float("inf")


# ------------------------------------------------------------------ gradients
@pytest.mark.parametrize("layout,R,scale", [(0, 64, 1.0), (1, 32, 1.3), (0, 48, 0.7)])
def test_gradients_by_formula_and_by_differences(layout, R, scale):
    rng = np.random.default_rng(R)
    B, H, T, D = 2, 3, 17, 64
    f, _ = mala.rope_frequencies(R, device="cuda")
    fn, pos = f.cpu().numpy(), rng.integers(0, 5000, (B, T))
    p = torch.from_numpy(pos).int().cuda()
    x, g = rows(rng, B, H, T, D, F32), rows(rng, B, H, T, D, F32)
    got = mala.rope_bwd(g, g[:, :1], p, f, layout, scale)
    check(got["dq"], g, pos, fn, layout, scale, True)
    check(got["dk"], g[:, :1].contiguous(), pos, fn, layout, scale, True)
    half = mala.rope_bwd(g, None, p, f, layout, scale, grad_dtype=BF16)
    assert half["dk"] is None
    check(half["dq"], g, pos, fn, layout, scale, True)
    # the map is linear, so a difference quotient in 64 bits is the derivative to rounding:
    # <g, y(x + h e) - y(x)> / h for a few elements e
    x64, g64 = x.double().cpu().numpy(), g.double().cpu().numpy()
    at = rng.integers(0, x64.size, 40)
    tol = bu.turned_bound(g64, fn, layout, scale, False, 5000)
    for i in at:
        e = np.zeros(x64.size)
        e[i] = 1.0
        e = e.reshape(x64.shape)
        d = (bu.turned(x64 + 0.5 * e, pos[:, None], fn, layout, scale)
             - bu.turned(x64 - 0.5 * e, pos[:, None], fn, layout, scale))
        want = float((g64 * d).sum())
        assert abs(want - float(got["dq"].flatten()[int(i)])) <= tol.flat[i] + 1e-11


def test_backward_is_the_transpose_of_the_forward():
    # <g, rope(x)> = <rope_bwd(g), x>, both sides with the kernel's own results
    rng = np.random.default_rng(8)
    f, s = mala.rope_frequencies(128, factor=4.0, scaling="yarn", original_len=1000, device="cuda")
    x, g = rows(rng, 1, 4, 600, 128, F32), rows(rng, 1, 4, 600, 128, F32)
    y = mala.rope(x, None, None, f, scale=s, out_dtype=F32)["q"]
    dx = mala.rope_bwd(g, None, None, f, scale=s)["dq"]
    a, b = float((g.double() * y.double()).sum()), float((dx.double() * x.double()).sum())
    bound = float((np.abs(g.cpu().numpy()) * bu.turned_bound(x.double().cpu().numpy(), f.cpu().numpy(), 0, s,
                                                             False, 600)).sum())
    assert abs(a - b) <= 2 * bound


def test_with_the_attention_and_its_backward():
    # projections -> rope -> fwd -> bwd -> rope_bwd against the dense formula in 64 bits
    rng = np.random.default_rng(9)
    B, Hq, Hkv, T, D = 1, 4, 2, 130, 64
    f, _ = mala.rope_frequencies(D, device="cuda")
    q, k, v = (rows(rng, B, h, T, D, BF16, "tokens") for h in (Hq, Hkv, Hkv))
    do = rows(rng, B, Hq, T, D, BF16)
    t = mala.rope(q, k, None, f)
    v = v.contiguous()
    scale = D ** -0.5
    fw = mala.fwd(t["q"], t["k"], v, scale, 0.0)
    bw = mala.bwd(t["q"], t["k"], v, fw["o"], fw["lse"], do, scale, 0.0)
    got = mala.rope_bwd(bw["dq"], bw["dk"], None, f)

    def leaf(x):
        return x.double().cpu().requires_grad_()

    qd, kd = leaf(t["q"]), leaf(t["k"])       # the rounded inputs of the attention
    s = qd @ kd.repeat_interleave(2, 1).transpose(2, 3).contiguous() * scale
    s = s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), float("-inf"))
    o = s.softmax(-1) @ v.double().cpu().repeat_interleave(2, 1)
    o.backward(do.double().cpu())
    for g, leaf_g in ((got["dq"], qd.grad), (got["dk"], kd.grad)):
        want = bu.turned(leaf_g.numpy(), np.arange(T), f.cpu().numpy(), 0, 1.0, True)
        # the attention's own bar for gradients (1e-2), of both elements of a pair: |cos| + |sin| of it
        assert np.abs(g.double().cpu().numpy() - want).max() <= 2 ** 0.5 * 1e-2


# ------------------------------------------------------------------ streams, graphs
def test_streams_and_current_device():
    rng = np.random.default_rng(10)
    f, _ = mala.rope_frequencies(128, device="cuda")
    x = [rows(rng, 1, 8, 500, 128, BF16) for _ in range(3)]
    want = [mala.rope(y, None, None, f)["q"] for y in x]
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = [mala.rope(y, None, None, f, stream=s)["q"] for y, s in zip(x, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_with_an_eager_call_alive():
    # forward and backward in a graph beside eager results of the same tensors, replayed with new
    # positions and inputs
    rng = np.random.default_rng(11)
    f, _ = mala.rope_frequencies(64, device="cuda")
    x, pos = rows(rng, 2, 4, 90, 64, BF16), torch.zeros((2, 90), dtype=torch.int32, device="cuda")
    eager = mala.rope(x, x[:, :2], pos, f)
    y, z = torch.empty_like(x), torch.empty(x.shape, device="cuda")

    def step():
        mala.mala_rope(x, None, y, None, pos, f, mala.ROPE_INTERLEAVED)
        mala.mala_rope(y, None, y, None, pos, f, mala.ROPE_INTERLEAVED, inverse=True)
        mala.mala_rope(y, None, z, None, pos, f)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape)))
        pos.copy_(torch.from_numpy(rng.integers(0, 1 << 20, (2, 90))))
        step()
        want = y.clone(), z.clone()
        torch.cuda.synchronize()
        y.zero_(), z.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(z, want[1])
        # there and back: three roundings to bf16 (in, out, back) of values up to |a| + |b|
        assert (y.float() - x.float()).abs().max() <= 3 * bu.U_BF16 * 2 * x.float().abs().max()
    assert eager["k"].shape == (2, 2, 90, 64)


def test_refusals_of_the_binding():
    f, _ = mala.rope_frequencies(64, device="cuda")
    q = torch.zeros((2, 4, 10, 64), dtype=BF16, device="cuda")
    o, p = torch.empty_like(q), torch.zeros(10, dtype=torch.int32, device="cuda")
    k = q[:, :2].contiguous()
    bad = [
        (TypeError, (q.half(), None, o, None, p, f)), (TypeError, (q, None, o.half(), None, p, f)),
        (TypeError, (q, None, None, None, p, f)), (ValueError, (q, None, o[:, :3], None, p, f)),
        (TypeError, (q, k.float(), o, k, p, f)), (ValueError, (q, k[:1], o, k[:1], p, f)),
        (ValueError, (q, k[..., :32], o, k[..., :32], p, f)), (ValueError, (q, None, o, k, p, f)),
        (ValueError, (q, k, o, None, p, f)), (ValueError, (q, None, o, None, p[:9], f)),
        (TypeError, (q, None, o, None, p.long(), f)), (ValueError, (q, None, o, None, p.expand(3, 10), f)),
        (TypeError, (q, None, o, None, p, f.float())), (TypeError, (q, None, o, None, p, None)),
        (TypeError, (q, None, o, None, p.cpu(), f)), (TypeError, (q, None, o, None, p, f.cpu())),
        (TypeError, (q.cpu(), None, o, None, p, f)), (TypeError, (q, None, o.cpu(), None, p, f)),
        (ValueError, (q.transpose(2, 3), None, q.transpose(2, 3), None, None, f)),
        (mala.MalaError, (q[..., :48], None, o[..., :48], None, p, f)),
        (mala.MalaError, (q, None, o, None, p, f[:12])), (mala.MalaError, (q, None, o, None, p, f, 2)),
        (mala.MalaError, (q, None, o, None, p, f, 0, float("nan"))),
        (mala.MalaError, (q, None, o, None, p, torch.cat([f, f])))]
    for err, args in bad:
        with pytest.raises(err):
            mala.mala_rope(*args)
