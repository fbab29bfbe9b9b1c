"""Plain 64-bit forms of the paged KV cache operators, and inputs for their tests."""
import math

import numpy as np
import torch

import oracle

U24 = 2.0 ** -24     # half a step of fp32, relative


def pages_of(n, P):
    return -(-n // P)


def pool(num_pages, Hkv, P, D, e4m3=False, layout="hpd", device="cuda"):
    """Zeroed k, v [num_pages, Hkv, P, D]: head-major pages of their own tensors, token-major
    ones with K and V of a page side by side, or every other head of a wider tensor."""
    dtype = torch.uint8 if e4m3 else torch.bfloat16
    if layout == "phd":
        both = torch.zeros((num_pages, 2, P, Hkv, D), dtype=dtype, device=device)
        k, v = both[:, 0].permute(0, 2, 1, 3), both[:, 1].permute(0, 2, 1, 3)
    elif layout == "wide":
        both = torch.zeros((num_pages, 2 * Hkv, P, 2 * D), dtype=dtype, device=device)
        k, v = both[:, ::2, :, :D], both[:, 1::2, :, D:]
    else:
        k = torch.zeros((num_pages, Hkv, P, D), dtype=dtype, device=device)
        v = torch.zeros_like(k)
    return (k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)) if e4m3 else (k, v)


def raw(t):
    """The same memory in a type that indexing takes."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def quarters(rng, shape, most=8):
    """Multiples of 1/4 up to most / 4: products of two of them are multiples of 1/16, so
    sums of 128 products are exact in fp32 (13 bits), and all are exact in bf16 and e4m3."""
    return torch.from_numpy(rng.integers(-most, most + 1, shape) / 4.0)


def scatter_tables(rng, lens, P, spare=3, width=None):
    """Table [S, W] (numpy int32, -1 behind a sequence's pages) and the pool's page count."""
    used = [pages_of(n, P) for n in lens]
    W = width or max(1, max(used))
    total = sum(used) + spare
    perm = rng.permutation(total)
    table = np.full((len(lens), W), -1, dtype=np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at:at + u]
        at += u
    return table, total


def fill(pool_t, table, lens, values, P):
    """values[b]: [Hkv, n_b, D] (float64, exact in the pool's type) into the pages."""
    r = raw(pool_t)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        x = values[b].to(torch.float32).to(pool_t.dtype)
        x = raw(x).to(pool_t.device)
        pos = torch.arange(n)
        page = torch.from_numpy(table[b].astype(np.int64))[pos // P]
        ok = page >= 0
        r[page[ok].to(r.device), :, (pos % P)[ok].to(r.device)] = x.transpose(0, 1)[ok.to(r.device)]


def decode_seq(q, k, v, seen, scale, tau, split, L):
    """One sequence in 64 bits by definition: q [Hq, D], k, v [Hkv, n, D], seen [n] bool.
    Returns o [Hq, D], lse [Hq], tiles [Hq], keep [Hq, tiles], tie (smallest |T / tau - 1|)."""
    Hq, D = q.shape
    Hkv, n, _ = k.shape
    g = Hq // Hkv
    nt = -(-n // 32)
    o, lse = np.zeros((Hq, D)), np.full(Hq, -math.inf)
    tiles, keep = np.zeros(Hq, dtype=np.int64), np.zeros((Hq, max(nt, 1)), dtype=bool)
    tie = np.full(Hq, math.inf)
    for h in range(Hq):
        s = (k[h // g] @ q[h]) * scale
        s[~seen] = -math.inf
        for lo in range(0, nt, split // 32):
            m, l = -math.inf, 0.0
            for t in range(min(nt, lo + split // 32) - 1, lo - 1, -1):
                x = s[32 * t:32 * t + 32]
                if not seen[32 * t:32 * t + 32].any():
                    continue
                mt = x.max()
                if l > 0 and tau > 0:
                    T = L * math.exp(mt - m - math.log(l))
                    tie[h] = min(tie[h], abs(T / tau - 1))
                    if T < tau:
                        continue
                keep[h, t] = True
                new = max(m, mt)
                if new > -math.inf:      # (a tile of scores of -inf adds nothing)
                    l = l * math.exp(m - new) + np.exp(x - new).sum()
                m = new
        s[~np.repeat(keep[h, :nt], 32)[:n]] = -math.inf
        tiles[h] = keep[h].sum()
        m = s.max(initial=-math.inf)
        if tiles[h] and m != -math.inf:
            p = np.exp(s - m)
            lse[h] = m + math.log(p.sum())
            o[h] = p @ v[h // g] / p.sum()
    return o, lse, tiles, keep, tie


def decode_bounds(n, smax, vmax, out_bf16):
    """Largest errors of (o, lse) for scores that are exact up to the scale.

    A score is rounded when it is scaled (twice: scale * log2 e, and the product), and its
    difference from the maximum once: 3 half steps of |s|, at most 2 smax apart; the
    exponential and its argument's range reduction add 2 steps.  The normaliser sums n terms
    (rescaled once per tile), the accumulator 3 n (three bf16 terms of every probability, 24
    bits).  lse takes the normaliser's relative error, the error of the maximum and of the
    logarithm; o both sums' relative errors, times at most vmax."""
    p = 3 * U24 * 2 * smax + 4 * U24
    s = (n + n // 32 + 8) * U24
    o = (2 * p + s + (3 * n + 16) * U24 + 2.0 ** -23) * vmax
    lse = p + s + 6 * U24 * (smax + math.log(max(n, 2)) + 1)
    return (o + 2.0 ** -8 * vmax if out_bf16 else o), lse


def update_plain(lens, new_lens, table, ring, state, P, num_pages, max_tokens):
    """A step's page tables with loops (all numpy; table and ring are changed in place)."""
    R, W = table.shape
    C = len(ring)
    head, count = min(max(int(state[0]), 0), C - 1), min(max(int(state[1]), 0), C)
    lens_out, cu = np.zeros(R, np.int32), np.zeros(R + 1, np.int32)
    slots, positions = np.full(max_tokens, -1, np.int32), np.zeros(max_tokens, np.int32)
    asked, taken, refused, given = 0, 0, 0, []
    popped = [int(ring[(head + i) % C]) for i in range(count)]
    for r in range(R):
        old, new = (min(max(int(x[r]), 0), W * P) for x in (lens, new_lens))
        have, want = pages_of(old, P), pages_of(new, P)
        need = max(0, want - have)
        ok = need == 0 or asked + need <= count
        for j in range(want, have):
            given.append(int(table[r, j]))
        if ok and need:
            table[r, have:want] = popped[asked:asked + need]
            taken = asked + need
        asked += need
        refused += not ok
        lens_out[r] = new if ok else old
        cu[r + 1] = cu[r] + max(0, new - old)
        for i, pos in enumerate(range(old, new)):
            t = cu[r] + i
            if t < max_tokens:
                page = int(table[r, pos // P])
                slots[t] = page * P + pos % P if ok and 0 <= page < num_pages else -1
                positions[t] = pos
    for i, page in enumerate(given):
        if i < C - count:
            ring[(head + count + i) % C] = page
    out = np.array([(head + taken) % C, count - taken + min(len(given), C - count), refused,
                    cu[R]], np.int32)
    return lens_out, cu, slots, positions, out


def e4m3_of(x, scale):
    """fp32 quotient, limited to +-448 (NaN stays), rounded to e4m3: as torch rounds on the CPU."""
    y = (x.to(torch.float32) / scale.to(torch.float32))
    return torch.where(y.isnan(), y, y.clamp(-448.0, 448.0)).to(torch.float8_e4m3fn)


def set_hash(keep, b, h):
    """The library's fingerprint of the retained tiles of head h of sequence b."""
    mask = (1 << 64) - 1
    total = 0
    for j in np.nonzero(keep)[0]:
        z = ((b << 52) | (h << 40) | int(j)) + 0x9E3779B97F4A7C15 & mask
        z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9 & mask
        z = (z ^ (z >> 27)) * 0x94D049BB133111EB & mask
        total = total + (z ^ (z >> 31)) & mask
    return total


def oracle_decode(q, k, v, scale, tau, splits):
    """The oracle's decode of one sequence (batch of one)."""
    return oracle.mala_decode(q[None], k[None], v[None], scale, tau, 32, splits)
