"""Plain 64-bit forms of rotary positions and of the cache with a scale per block, for tests."""
import math

import numpy as np
import torch

import paged_util as pu

E_MIN, E_MAX = -117, 120
U_BF16 = 2.0 ** -8       # half a step of bf16, relative


# ------------------------------------------------------------------ rotary positions
def turned(x, pos, inv_freq, layout, scale, inverse=False):
    """x [..., T, D] float64 at positions [..., T]: pair by pair, as defined."""
    R = 2 * len(inv_freq)
    theta = pos[..., None].astype(np.float64) * inv_freq
    c, s = np.cos(theta), np.sin(theta) * (-1.0 if inverse else 1.0)
    y = x.copy()
    a, b = (np.arange(R // 2), np.arange(R // 2) + R // 2) if layout == 0 else \
        (np.arange(0, R, 2), np.arange(1, R, 2))
    y[..., a] = scale * (x[..., a] * c - x[..., b] * s)
    y[..., b] = scale * (x[..., b] * c + x[..., a] * s)
    return y


def turned_bound(x, inv_freq, layout, scale, out_bf16, far):
    """Largest error of a turned element.

    cos and sin: the angle left of a quarter turn is rounded to fp32 (at most 2^-25 of an angle below
    1), the square of it once (half of it counts: 0.3 half steps), the last fused operation once
    (half a step of 1): 2 half steps in all, and one when the scale is multiplied in.  The product
    b sin is rounded once, the fused sum once.  So 5 half steps of (|a| + |b|) |scale|; the oracle's own
    angle is off by half a step of 2^-53 of it, and its cosine by as much."""
    R = 2 * len(inv_freq)
    size = np.abs(x).astype(np.float64)
    m = size.copy()
    a, b = (np.arange(R // 2), np.arange(R // 2) + R // 2) if layout == 0 else \
        (np.arange(0, R, 2), np.arange(1, R, 2))
    m[..., a] = m[..., b] = (size[..., a] + size[..., b]) * abs(scale)
    own = 4 * 2.0 ** -53 * max(far, 1) * max(float(np.abs(inv_freq).max()), 1.0)
    err = m * (5 * pu.U24 + own)
    err[..., R:] = 0.0
    return err + (U_BF16 * (m + err) if out_bf16 else pu.U24 * m)


# ------------------------------------------------------------------ blocks
def e4m3(y):
    """float64 rounded to e4m3 (nearest even, no limit applied: |y| at most 448)."""
    a = np.abs(y)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = np.where(a >= 2.0 ** -6, np.exp2(np.floor(np.log2(np.where(a > 0, a, 1.0))) - 3), 2.0 ** -9)
    return np.where(np.isnan(y), y, np.copysign(np.rint(a / step) * step, y))


def exponent(x):
    """The least e in range with |x| <= 448 2^e for the finite x."""
    x = np.abs(x[np.isfinite(x)])
    top = float(x.max()) if x.size else 0.0
    e = E_MIN
    while e < E_MAX and top > math.ldexp(448.0, e):
        e += 1
    return e


def write_plain(values, exps, new, slots):
    """new [H, T, D] float64 into values [N, H, P, D] (e4m3 values) and exps [N, H, P / 16], in place:
    block by block, as defined."""
    N, H, P, D = values.shape
    rows = {}
    for t, s in enumerate(slots):
        if 0 <= s < N * P:
            rows.setdefault(int(s) // 16, {})[int(s) % 16] = t
    for block, mine in rows.items():
        page, w = block // (P // 16), block % (P // 16)
        for h in range(H):
            x = new[h, list(mine.values())]
            e = exponent(x)
            old = min(max(int(exps[page, h, w]), E_MIN), E_MAX)
            span = values[page, h, 16 * w:16 * w + 16]
            if 0 not in mine:
                e = max(e, old)
                if e > old:
                    keep = [r for r in range(16) if r not in mine]
                    span[keep] = e4m3(span[keep] * 2.0 ** (old - e))
            exps[page, h, w] = e
            limit = 240.0 if e == E_MAX else 448.0
            y = np.ldexp(x, -e)
            span[list(mine.keys())] = e4m3(np.where(np.isnan(y), y, np.clip(y, -limit, limit)))


def as_bytes(values):
    """e4m3 values as bytes (uint8, CPU)."""
    return torch.from_numpy(values).float().to(torch.float8_e4m3fn).view(torch.uint8)


def same_bytes(got, want):
    """Equal bytes, any NaN for a NaN, and -0 for 0 (a value below half the smallest keeps its sign)."""
    nan = (want & 0x7F) == 0x7F
    return bool((((got & 0x7F) == 0x7F) == nan).all()) and bool((got[~nan] == want[~nan]).all())


def block_cache(mala, N, Hkv, P, D, layout="hpd", device="cuda", fill=0):
    """(cache, k, v, ks, vs): pages as pu.pool makes them, every byte `fill`."""
    k, v = pu.pool(N, Hkv, P, D, True, layout, device)
    ks, vs = (torch.full((N, Hkv, P // 16), fill, dtype=torch.uint8, device=device)
              .view(torch.float8_e8m0fnu) for _ in range(2))
    for t in (k, v):
        pu.raw(t).fill_(fill)
    return (mala.PagedCache(k, v, ks, vs) if mala else None), k, v, ks, vs


def held(t, exps):
    """float64 values x scales [N, H, P, D] of a cache's tensor on the CPU."""
    x = t.view(torch.uint8).cpu().contiguous().view(torch.float8_e4m3fn).float().double().numpy()
    e = exps.view(torch.uint8).cpu().numpy().astype(np.int64) - 127
    return x * np.exp2(np.repeat(e, 16, axis=2)[..., None].astype(np.float64))
