"""The calls around a cache in 8 bits whose speed matters: rotary positions of queries and keys
(and of their gradients), rows into pages that hold e4m3 values with a scale for every 16
tokens and head, both in one call, pages back to packed rows, and the decode over such pages.

Rotation: theta_i = position * inv_freq[i], i < R / 2; a pair (a, b) of the first R elements of
a row becomes scale * (a cos - b sin, b cos + a sin): "half" pairs elements i and i + R / 2,
"interleaved" 2 i and 2 i + 1.  Gradients take the transposed rotation.

Cache: 16 rows of a page from a multiple of 16 on, of one KV head, are a block: e4m3 values of
one scale 2^e, held as an 8-bit exponent, K and V apart.  e is the least integer with
amax <= 448 * 2^e of the new rows; a block whose row 0 is among them starts anew, any other
keeps its scale or takes the larger one, and then its other rows are rounded again.
With `own` the calls are the framework's; otherwise the same operators in torch.
"""
import math
import random

import torch

own = False

_TILE = 32           # keys per decision tile of the decode
_BLOCK = 16          # rows that share a scale
_E4M3_MAX = 448.0
_E_MIN, _E_MAX = -117, 120


# ------------------------------------------------------------------ the cases
def listed():
    rope = dict(kind="rope", B=1, layout="half", inverse=False, scale=1.0, src="tokens",
                dst="tokens", in_t="bf16", out_t="bf16")
    write = dict(P=16, pages="hpd", pad=0.0)
    dec = dict(kind="decode", tau=0.0, split=128, pages="hpd", out="bf16")
    return [
        # rope: queries and keys of a decode step, far positions; latency
        dict(rope, name="rope_decode_64", T=64, Hq=32, Hkv=8, D=128, R=128, far=131072),
        # rope: packed prompts of a small model, half of each head, interleaved pairs, from
        # projection rows to the packed layout of the attention
        dict(rope, name="rope_prompts_20000", T=20000, Hq=16, Hkv=4, D=64, R=32, far=0,
             layout="interleaved", dst="heads"),
        # rope: gradients of a training step's queries and keys, fp32 from the attention's
        # backward, bf16 for the projection's; frequencies scaled for a longer context
        dict(rope, name="rope_grads_2x8000", B=2, T=8000, Hq=32, Hkv=8, D=128, R=128, far=0,
             inverse=True, scale=1.2, src="heads", dst="heads", in_t="f32"),
        # write: the new tokens of a decode step, each into a block that holds others; latency
        dict(write, kind="write", name="write_decode_64", mix="decode", T=64, Hkv=8, D=128,
             src="tokens"),
        # write: prompts and chunks of prompts, padded to a captured step's size, into
        # token-major pages
        dict(write, kind="write", name="write_chunks_20000", mix="chunks", T=20000, Hkv=8, D=128,
             src="heads", P=32, pages="phd", pad=0.05),
        # rotated write: queries, keys and values of a decode step in one call
        dict(write, kind="rope_write", name="rope_write_decode_64", mix="decode", T=64, Hq=32,
             Hkv=8, D=128, R=128, layout="half", scale=1.0, src="tokens"),
        # rotated write: a prefill step of several chunks, part of each head rotated
        dict(write, kind="rope_write", name="rope_write_chunks_16000", mix="chunks", T=16000, Hq=32,
             Hkv=8, D=128, R=64, layout="half", scale=1.0, src="tokens", P=64),
        # read: the cached part of a few prompts of a chunked prefill
        dict(kind="read", name="read_6x700", S=6, Hkv=2, D=128, P=16, lens="uniform", n=700,
             pages="hpd"),
        # read: a prefill batch against long cached prefixes
        dict(kind="read", name="read_10x10000", S=10, Hkv=8, D=128, P=64, lens="uniform", n=10000,
             pages="hpd"),
        # decode: one short sequence, one tensor-parallel rank's heads; latency alone
        dict(dec, name="decode_1x300", B=1, Hq=8, Hkv=2, D=128, P=16, lens="full", n=300),
        # decode: a serving batch of ragged caches, tiles skipped by mass
        dict(dec, name="decode_48_ragged", B=48, Hq=32, Hkv=8, D=128, P=32, lens="uniform", n=8192,
             tau=1e-3, split=256),
        # decode: long caches; bandwidth, offsets past 32 bits of values
        dict(dec, name="decode_16x100k", B=16, Hq=32, Hkv=8, D=128, P=64, lens="full", n=100000),
    ]


def _logsize(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "write", "rope_write", "read", "decode", "decode"])
    Hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
    P = rng.choice([16, 16, 32, 48, 64, 128, 256])
    group = rng.choice([1, 2, 4, 4, 5, 7, 8])
    c = dict(kind=kind, lseed=rng.randrange(1 << 30), Hkv=Hkv, D=D)
    turn = dict(R=rng.choice([D, D, D, D // 2, D * 3 // 4, D // 4]),
                layout=rng.choice(["half", "half", "interleaved"]),
                scale=rng.choice([1.0, 1.0, 1.2, 0.75]))
    if kind == "rope":
        T = _logsize(rng, 1, 32768)
        return dict(c, **turn, Hq=Hkv * group, B=max(1, min(_logsize(rng, 1, 16), 32768 // T)), T=T,
                    far=rng.choice([0, 0, 131072, 1 << 24]), inverse=rng.random() < 0.4,
                    src=rng.choice(["tokens", "heads"]), dst=rng.choice(["tokens", "heads"]),
                    in_t=rng.choice(["bf16", "bf16", "f32"]),
                    out_t=rng.choice(["bf16", "bf16", "f32"]))
    c.update(P=P, pages=rng.choice(["hpd", "hpd", "phd"]))
    if kind in ("write", "rope_write"):
        mix = rng.choice(["decode", "chunks"])
        c.update(mix=mix, T=_logsize(rng, 1, 2048 if mix == "decode" else 32768),
                 src=rng.choice(["tokens", "heads"]), pad=rng.choice([0.0, 0.05, 0.4]))
        return dict(c, **turn, Hq=Hkv * group) if kind == "rope_write" else c
    lens = rng.choice(["full", "uniform", "log"])
    if kind == "read":
        n = _logsize(rng, 1, 16384)
        return dict(c, S=max(1, min(_logsize(rng, 1, 64), 131072 // n)), lens=lens, n=n)
    n = _logsize(rng, 1, 65536)
    return dict(c, B=max(1, min(_logsize(rng, 1, 128), 262144 // n)), Hq=Hkv * group, lens=lens, n=n,
                tau=rng.choice([0.0, 0.0, 1e-4, 1e-3]), split=rng.choice([128, 256, 512]),
                out=rng.choice(["bf16", "bf16", "f32"]))


def _lengths(case, count):
    """Lengths up to case["n"], a function of the case alone."""
    n, rng = case["n"], random.Random(case.get("lseed", 1))
    if case["lens"] == "full":
        return [n] * count
    if case["lens"] == "uniform":
        # (every eighth row of a batch is idle, just begun or as the others)
        return [rng.choice([0, 1, rng.randint(1, n)]) if i % 8 == 7 else rng.randint(1, n)
                for i in range(count)]
    return [_logsize(rng, 1, n) for _ in range(count)]


def _growth(case):
    """(tokens cached, new tokens) of each request of a step, from the case alone."""
    rng, left = random.Random(case.get("lseed", 1)), case["T"] - int(case["T"] * case["pad"])
    if case["mix"] == "decode":
        return [(rng.randint(1, 400), 1) for _ in range(max(1, left))]
    steps = []
    while left > 0:
        n = min(left, rng.randint(1, 4096))
        # a new prompt, or the next chunk of one that left its last block part full
        steps.append((rng.choice([0, 0, rng.randint(1, 400)]), n))
        left -= n
    return steps or [(0, 1)]


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _inv_freq(R, scaled):
    """Frequencies of base 10000; `scaled`: the slow ones divided by 8, a ramp between them."""
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    f = 10000.0 ** (-2.0 * i / R)
    if scaled:
        turns = 4096 * f / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * keep + f / 8.0 * (1.0 - keep)
    return f


def _rows(g, B, H, T, D, src, dtype):
    """[B, H, T, D] rows: contiguous ("heads"), or slices of [B, T, H, D] rows."""
    if src == "heads":
        return torch.randn((B, H, T, D), generator=g, device="cuda").to(dtype)
    return torch.randn((B, T, H, D), generator=g, device="cuda").to(dtype).transpose(1, 2)


def _pool(case, g, num_pages):
    """k, v as [num_pages, Hkv, P, D] views of e4m3 values, and their blocks' exponents
    [num_pages, Hkv, P / 16]: values of normals of about 1 in all."""
    Hkv, P, D = case["Hkv"], case["P"], case["D"]
    if case["pages"] == "phd":       # token-major pages, K and V of a page side by side
        both = torch.empty((num_pages, 2, P, Hkv, D), dtype=torch.float8_e4m3fn, device="cuda")
        k, v = both[:, 0].permute(0, 2, 1, 3), both[:, 1].permute(0, 2, 1, 3)
        fill = [both]
    else:
        k = torch.empty((num_pages, Hkv, P, D), dtype=torch.float8_e4m3fn, device="cuda")
        v = torch.empty_like(k)
        fill = [k, v]
    for t in fill:
        flat, step = t.view(-1), 1 << 27
        for i in range(0, flat.numel(), step):
            part = flat[i:i + step]
            x = torch.randn(part.numel(), generator=g, device="cuda") * 64
            part.copy_(x.clamp_(-_E4M3_MAX, _E4M3_MAX))
    shape = (num_pages, Hkv, P // _BLOCK)
    ks, vs = (torch.randint(120, 123, shape, generator=g, device="cuda").to(torch.uint8)
              .view(torch.float8_e8m0fnu) for _ in range(2))
    return k, v, ks, vs


def _tables(case, g, lens):
    """Scattered pages for sequences of these lengths: (table [S, W], pages in the pool)."""
    P, W = case["P"], max(1, -(-max(lens) // case["P"]))
    used = torch.tensor([-(-n // P) for n in lens], device="cuda")
    total = int(used.sum())
    pool = total + max(1, total // 8)
    perm = torch.randperm(pool, generator=g, device="cuda").int()
    j = torch.arange(W, device="cuda")
    at = ((used.cumsum(0) - used)[:, None] + j).clamp_(max=pool - 1)
    return torch.where(j < used[:, None], perm[at], -1).int().contiguous(), pool


def prepare(case, seed):
    g = _gen(seed)
    kind, s = case["kind"], dict(case=case)
    D, Hkv = case["D"], case["Hkv"]
    if kind == "rope":
        B, T, Hq = case["B"], case["T"], case["Hq"]
        t_in, t_out = _type(case["in_t"]), _type(case["out_t"])
        for name, H in (("q", Hq), ("k", Hkv)):
            s[name] = _rows(g, B, H, T, D, case["src"], t_in)
            shape = (B, H, T, D) if case["dst"] == "heads" else (B, T, H, D)
            out = torch.empty(shape, dtype=t_out, device="cuda")
            s[name + "_out"] = out if case["dst"] == "heads" else out.transpose(1, 2)
        if case["far"]:
            s["pos"] = torch.randint(case["far"], (B, T), generator=g, device="cuda").int()
        else:                                # sequences of 1500 tokens, one after the other
            s["pos"] = (torch.arange(T, device="cuda") % 1500).int().expand(B, T).contiguous()
        s["inv_freq"] = _inv_freq(case["R"], case["scale"] != 1.0)
        return s
    if kind in ("write", "rope_write"):
        steps, T = _growth(case), case["T"]
        s["table"], pages = _tables(case, g, [a + n for a, n in steps])
        old, n = (torch.tensor(x, device="cuda") for x in zip(*steps))
        end = n.cumsum(0)
        t = torch.arange(T, device="cuda")
        r = torch.searchsorted(end, t, right=True).clamp(max=len(steps) - 1)
        live = t < end[-1]
        pos = torch.where(live, old[r] + t - (end - n)[r], 0)
        page = s["table"][r, (pos // case["P"]).clamp(max=s["table"].shape[1] - 1)]
        s["slots"] = torch.where(live, page * case["P"] + pos % case["P"], -1).int()
        s["k"], s["v"], s["ks"], s["vs"] = _pool(case, g, pages)
        new = _rows(g, 2, Hkv, T, D, "heads", torch.bfloat16) if case["src"] == "heads" else \
            torch.randn((T, 2, Hkv, D), generator=g, device="cuda").bfloat16().permute(1, 2, 0, 3)
        s["k_new"], s["v_new"] = new[0], new[1]
        if kind == "rope_write":
            s["pos"] = pos.int()
            s["inv_freq"] = _inv_freq(case["R"], case["scale"] != 1.0)
            s["q"] = _rows(g, 1, case["Hq"], T, D, case["src"], torch.bfloat16)[0]
            # a decode takes [T, Hq, D] queries, a prefill [Hq, T, D]
            shape = (T, case["Hq"], D) if case["mix"] == "decode" else (case["Hq"], T, D)
            out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
            s["q_out"] = out.transpose(0, 1) if case["mix"] == "decode" else out
    else:
        lens = _lengths(case, case["S"] if kind == "read" else case["B"])
        s["table"], pages = _tables(case, g, lens)
        s["k"], s["v"], s["ks"], s["vs"] = _pool(case, g, pages)
        s["max_len"] = max(max(lens), 1)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        if kind == "read":
            s["cu"] = torch.nn.functional.pad(s["lens"].cumsum(0), (1, 0)).int()
            s["total"] = max(1, sum(lens))
            s["k_out"] = torch.zeros((Hkv, s["total"], D), dtype=torch.bfloat16, device="cuda")
            s["v_out"] = torch.zeros_like(s["k_out"])
        else:
            # queries that look for the sum of the keys at four places, and noise
            B, Hq, P = case["B"], case["Hq"], case["P"]
            q = torch.randn((B, Hq, D), generator=g, device="cuda")
            head = torch.arange(Hq, device="cuda") // (Hq // Hkv)
            for _ in range(4):
                at = torch.rand((B, Hq), generator=g, device="cuda")
                at = (at * s["lens"][:, None]).long().clamp_(min=0)
                page = s["table"].gather(1, (at // P).clamp_(max=s["table"].shape[1] - 1))
                page, row = page.long().clamp_(min=0), at % P
                x = s["k"].view(torch.uint8)[page, head.expand(B, Hq), row]
                x = x.view(torch.float8_e4m3fn).float()
                x *= _powers(s["ks"])[page, head.expand(B, Hq), row // _BLOCK][..., None]
                q += x * (3.0 if case["tau"] > 0 else 1.0)
            s["q"] = q.bfloat16()
            s["scale"] = D ** -0.5
            s["o"] = torch.empty((B, Hq, D), dtype=_type(case["out"]), device="cuda")
            s["lse"] = torch.empty((B, Hq), dtype=torch.float32, device="cuda")
    if own:      # what a serving program makes once: the handle of its cache, a workspace
        import paper_2609_32712_amd as mala
        s["cache"] = mala.PagedCache(s["k"], s["v"], s["ks"], s["vs"])
        if kind == "decode":
            need = mala.mala_paged_decode_workspace_size(case["B"], case["Hq"], Hkv, D, s["max_len"],
                                                         case["split"])
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _powers(exponents):
    """fp32 2^e of stored exponents."""
    return torch.exp2(exponents.view(torch.uint8).float() - 127.0)


# ------------------------------------------------------------------ one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"rope": _own_rope, "write": _own_write, "rope_write": _own_rope_write,
                "read": _own_read, "decode": _own_decode}[kind](s)
    return {"rope": _plain_rope, "write": _plain_write, "rope_write": _plain_rope_write,
            "read": _plain_read, "decode": _plain_decode}[kind](s)


def _layout(mala, case):
    return mala.ROPE_HALF if case["layout"] == "half" else mala.ROPE_INTERLEAVED


def _own_rope(s):
    import paper_2609_32712_amd as mala
    c = s["case"]
    mala.mala_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["pos"], s["inv_freq"],
                   _layout(mala, c), c["scale"], inverse=c["inverse"])
    return [s["q_out"], s["k_out"]]


def _own_write(s):
    import paper_2609_32712_amd as mala
    mala.mala_paged_write(s["k_new"], s["v_new"], s["slots"], s["cache"])
    return [s["k"], s["v"], s["ks"], s["vs"]]


def _own_rope_write(s):
    import paper_2609_32712_amd as mala
    c = s["case"]
    mala.mala_paged_rope_write(s["q"], s["q_out"], s["k_new"], s["v_new"], s["pos"], s["slots"],
                               s["cache"], s["inv_freq"], _layout(mala, c), c["scale"])
    return [s["q_out"], s["k"], s["v"], s["ks"], s["vs"]]


def _own_read(s):
    import paper_2609_32712_amd as mala
    mala.mala_paged_read(s["cache"], s["table"], s["cu"], s["max_len"], s["k_out"], s["v_out"])
    return [s["k_out"], s["v_out"]]


def _own_decode(s):
    import paper_2609_32712_amd as mala
    c = s["case"]
    mala.mala_paged_decode(s["q"], s["cache"], s["table"], s["lens"], s["max_len"], s["o"],
                           s["lse"], None, None, c["split"], s["workspace"], s["scale"], c["tau"])
    return [s["o"], s["lse"]]


def _turned(x, pos, inv_freq, layout, scale, inverse):
    """fp32 rows [..., T, D] rotated by their positions [..., T]."""
    R = 2 * inv_freq.numel()
    angle = pos.double()[..., None] * inv_freq
    cos, sin = angle.cos().float() * scale, angle.sin().float() * scale
    if inverse:
        sin = -sin
    x = x.float()
    y = x.clone()
    if layout == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_rope(s):
    c = s["case"]
    for x, out in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
        out.copy_(_turned(x, s["pos"][:, None], s["inv_freq"], c["layout"], c["scale"],
                          c["inverse"]))
    return [s["q_out"], s["k_out"]]


def _into_blocks(pool, exponents, new, slots):
    """Rows new [Hkv, T, D] (bf16) into a pool of e4m3 values and its exponents, in place."""
    pages, H, P, D = pool.shape
    per_page = P // _BLOCK
    # tokens without a slot go to one page more than there are
    good = (slots >= 0) & (slots < pages * P)
    slot = torch.where(good, slots, pages * P).long()
    block = slot // _BLOCK
    x = new.transpose(0, 1).float()
    size = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)                     # [T, H]
    blocks = (pages + 1) * per_page
    top = torch.zeros((blocks, H), device="cuda").scatter_reduce_(
        0, block[:, None].expand(-1, H), size, "amax")
    touched = torch.zeros(blocks, dtype=torch.bool, device="cuda")
    touched[block] = True
    fresh = torch.zeros(blocks, dtype=torch.bool, device="cuda")
    fresh[block[slot % _BLOCK == 0]] = True
    m, ex = torch.frexp(top)
    e_new = torch.where(top > 0, ex - 9 + (m > 0.875).int(), _E_MIN).clamp(_E_MIN, _E_MAX)
    e_new = e_new[:-per_page].view(pages, per_page, H).transpose(1, 2)
    touched, fresh = (z[:-per_page].view(pages, 1, per_page) for z in (touched, fresh))
    byte = exponents.view(torch.uint8)
    e_old = byte.int().clamp(127 + _E_MIN, 127 + _E_MAX) - 127
    e = torch.where(fresh, e_new, torch.maximum(e_old, e_new))
    # other rows of a block whose scale grows: rounded again
    less = torch.where(touched & ~fresh, (e_old - e).float(), 0.0)
    rows = pool.float().reshape(pages, H, per_page, _BLOCK, D)
    rows = (rows * torch.exp2(less)[..., None, None]).view(pages, H, P, D)
    longer = torch.cat([rows, rows[:1]])
    e_row = torch.cat([e, e[:1]])[slot // P, :, slot % P // _BLOCK]            # [T, H]
    most = torch.where(e_row == _E_MAX, 240.0, _E4M3_MAX)[..., None]
    y = (x.double() * torch.exp2(-e_row.double())[..., None]).float()
    longer[slot // P, :, slot % P] = torch.where(y.isnan(), y, torch.minimum(torch.maximum(y, -most), most))
    pool.copy_(longer[:pages].to(pool.dtype))
    byte.copy_(torch.where(touched, e + 127, byte.int()).to(torch.uint8))


def _plain_write(s):
    _into_blocks(s["k"], s["ks"], s["k_new"], s["slots"])
    _into_blocks(s["v"], s["vs"], s["v_new"], s["slots"])
    return [s["k"], s["v"], s["ks"], s["vs"]]


def _plain_rope_write(s):
    c = s["case"]
    turn = (s["pos"], s["inv_freq"], c["layout"], c["scale"], False)
    s["q_out"].copy_(_turned(s["q"], *turn))
    # (the key as a bf16, as the attention of a prompt takes it)
    _into_blocks(s["k"], s["ks"], _turned(s["k_new"], *turn).bfloat16(), s["slots"])
    _into_blocks(s["v"], s["vs"], s["v_new"], s["slots"])
    return [s["q_out"], s["k"], s["v"], s["ks"], s["vs"]]


def _plain_read(s):
    P, lens = s["case"]["P"], s["lens"]
    width = -(-s["max_len"] // P)
    t = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(s["cu"][1:], t.int(), right=True).clamp(max=lens.numel() - 1)
    pos = t - s["cu"][seq].long()
    page = s["table"][seq, (pos // P).clamp(max=width - 1)].long().clamp(min=0)
    for pool, exponents, out in ((s["k"], s["ks"], s["k_out"]), (s["v"], s["vs"], s["v_out"])):
        x = pool.view(torch.uint8)[page, :, pos % P].view(pool.dtype).float()
        x = x * _powers(exponents)[page, :, pos % P // _BLOCK][..., None]
        out.copy_(torch.where((t < s["cu"][-1])[:, None], x.transpose(0, 1), out))
    return [s["k_out"], s["v_out"]]


def _gathered(pool, exponents, table, width):
    """[S, Hkv, width * P, D] fp32 rows of the first `width` pages of each table row."""
    at = table[:, :width].long().clamp(min=0)
    raw = pool.view(torch.uint8)[at].permute(0, 2, 1, 3, 4)
    S, H, W, P, D = raw.shape
    x = raw.reshape(S, H, W * P // _BLOCK, _BLOCK, D).view(pool.dtype).float()
    x *= _powers(exponents)[at].permute(0, 2, 1, 3).reshape(S, H, W * P // _BLOCK, 1, 1)
    return x.reshape(S, H, W * P, D)


def _plain_decode(s):
    case, table, lens = s["case"], s["table"], s["lens"]
    B, Hq, Hkv, D, P = case["B"], case["Hq"], case["Hkv"], case["D"], case["P"]
    width = -(-s["max_len"] // P)
    N = width * P
    k = _gathered(s["k"], s["ks"], table, width)
    score = torch.matmul(s["q"].float().view(B, Hkv, Hq // Hkv, D), k.transpose(2, 3)) * s["scale"]
    del k
    pos = torch.arange(N, device="cuda")
    seen = (pos < lens[:, None]) & (table[:, :width] >= 0).repeat_interleave(P, 1)
    score = score.masked_fill(~seen[:, None, None], -math.inf).view(B, Hq, N)
    if case["tau"] > 0:
        score = score.masked_fill(~_retained(score, lens, case["tau"], case["split"]), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    v = _gathered(s["v"], s["vs"], table, width)
    o = torch.matmul(p.view(B, Hkv, Hq // Hkv, N), v).view(B, Hq, D)
    o = torch.where(total > 0, o / total, 0.0)
    return [o.to(s["o"].dtype), (top + torch.log(total)).squeeze(-1)]


def _retained(score, lens, tau, split):
    """The keys whose tile of 32 is retained: in each run of `split` keys, from its last tile
    down, a tile is left out when its largest score is below the log-sum of those kept so far
    by more than log(n / tau).  (Whether a tile is kept depends on the ones before it: a loop
    over the tiles of a run, all runs at once.)"""
    B, Hq, N = score.shape
    runs, tiles = -(-N // split), split // _TILE
    x = torch.nn.functional.pad(score, (0, runs * split - N), value=-math.inf)
    x = x.view(B, Hq, runs, tiles, _TILE)
    best = x.amax(-1)
    sums = torch.exp(x - torch.where(best > -math.inf, best, 0.0)[..., None]).sum(-1)
    limit = math.log(tau) - torch.log(lens.float().clamp(min=1))[:, None, None]
    m = torch.full((B, Hq, runs), -math.inf, device="cuda")
    z = torch.zeros_like(m)
    keep = torch.zeros((B, Hq, runs, tiles), dtype=torch.bool, device="cuda")
    for j in range(tiles - 1, -1, -1):
        b = best[..., j]
        take = (b > -math.inf) & ((z == 0) | (b - m - torch.log(z) >= limit))
        new = torch.maximum(m, b)
        shift = torch.where(new > -math.inf, new, 0.0)
        both = z * torch.exp(m - shift) + sums[..., j] * torch.exp(b - shift)
        z, m = torch.where(take, both, z), torch.where(take, new, m)
        keep[..., j] = take
    return keep[..., None].expand(x.shape).reshape(B, Hq, runs * split)[..., :N]


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, D, Hkv = case["kind"], case["D"], case["Hkv"]
    size = {"bf16": 2, "f32": 4}
    if kind == "rope":
        values = case["B"] * case["T"] * (case["Hq"] + Hkv) * D
        turned = values // D * case["R"]
        return dict(bytes=values * (size[case["in_t"]] + size[case["out_t"]])
                    + case["B"] * case["T"] * 4 + case["R"] * 4, flops=3 * turned)
    if kind in ("write", "rope_write"):
        steps = _growth(case)
        tokens = sum(n for _, n in steps)
        blocks = sum(-(-(a + n) // _BLOCK) - a // _BLOCK for a, n in steps)
        moved = tokens * 2 * Hkv * D * 3 + blocks * 2 * Hkv + case["T"] * 4
        if kind == "write":
            return dict(bytes=moved, flops=2 * tokens * 2 * Hkv * D)
        rows = case["T"] * case["Hq"]
        return dict(bytes=moved + rows * D * 4 + case["T"] * 4 + case["R"] * 4,
                    flops=3 * (rows + tokens * Hkv) * case["R"] + 2 * tokens * 2 * Hkv * D)
    lens = _lengths(case, case["S"] if kind == "read" else case["B"])
    pages = sum(-(-n // case["P"]) for n in lens)
    blocks = sum(-(-n // _BLOCK) for n in lens)
    held = sum(lens) * 2 * Hkv * D + blocks * 2 * Hkv + 4 * pages
    if kind == "read":
        return dict(bytes=held + sum(lens) * 2 * Hkv * D * 2, flops=sum(lens) * 2 * Hkv * D)
    ends = case["B"] * case["Hq"] * (D * (2 + size[case["out"]]) + 4)
    return dict(bytes=held + ends, flops=4 * sum(lens) * case["Hq"] * D)


# ------------------------------------------------------------------ the definition in 64 bits
def _rotate_exact(x, pos, case):
    """Rows [..., T, D] in 64 bits, as complex numbers times e^(i theta)."""
    R, s = case["R"], case["scale"]
    f = _inv_freq(R, s != 1.0)
    theta = pos.double()[..., None] * f * (-1.0 if case.get("inverse") else 1.0)
    x = x.double()
    part = x[..., :R]
    if case["layout"] == "half":
        z = torch.complex(part[..., :R // 2].contiguous(), part[..., R // 2:].contiguous())
    else:
        z = torch.view_as_complex(part.reshape(*part.shape[:-1], R // 2, 2).contiguous())
    z = z * torch.polar(torch.full_like(theta, s), theta)
    turned = torch.cat([z.real, z.imag], -1) if case["layout"] == "half" else \
        torch.view_as_real(z).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1)


def _blocks_exact(pool, exponents, new, slots):
    """Values over their scales, before the last rounding, and the scales: [pool, scales]."""
    pages, H, P, D = pool.shape
    rows = pool.float().double().permute(0, 2, 1, 3).reshape(pages * P, H, D)
    held = exponents.view(torch.uint8).double().sub(127).clamp(_E_MIN, _E_MAX)
    held = held.permute(0, 2, 1).reshape(-1, H)
    hit = ((slots >= 0) & (slots < pages * P)).nonzero().view(-1)
    slot = slots[hit].long()
    x = new.double().transpose(0, 1)[hit]
    row_e = torch.where(x.abs() > 0, torch.ceil(torch.log2(x.abs() / _E4M3_MAX)), _E_MIN)
    # (the least e with |x| <= 448 2^e; log2 alone may be off next to a power)
    row_e = torch.where(x.abs() > _E4M3_MAX * torch.exp2(row_e), row_e + 1, row_e)
    row_e = torch.where(x.abs() <= _E4M3_MAX * torch.exp2(row_e - 1), row_e - 1, row_e)
    row_e = row_e.amax(-1).clamp(_E_MIN, _E_MAX)
    order = torch.argsort(slot // _BLOCK, stable=True)
    ids, counts = torch.unique_consecutive((slot // _BLOCK)[order], return_counts=True)
    which = torch.repeat_interleave(torch.arange(ids.numel(), device="cuda"), counts)
    e = torch.full((ids.numel(), H), float(_E_MIN), dtype=torch.float64, device="cuda")
    e.index_reduce_(0, which, row_e[order], "amax")
    begun = torch.zeros(ids.numel(), dtype=torch.float64, device="cuda")
    begun.index_add_(0, which, (slot[order] % _BLOCK == 0).double())
    e = torch.where(begun[:, None] > 0, e, torch.maximum(e, held[ids]))
    rows = rows.view(-1, _BLOCK, H, D)
    rows[ids] = torch.where(begun[:, None, None, None] > 0, rows[ids],
                            rows[ids] * torch.exp2(held[ids] - e)[:, None, :, None])
    held[ids] = e
    rows = rows.view(pages * P, H, D)
    rows[slot] = x * torch.exp2(-held[slot // _BLOCK])[..., None]
    return rows.view(pages, P, H, D).permute(0, 2, 1, 3).contiguous(), \
        torch.exp2(held).view(pages, P // _BLOCK, H).permute(0, 2, 1).contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    kind, P, D = case["kind"], case["P"] if "P" in case else 0, case["D"]
    if kind == "rope":
        return [_rotate_exact(x, s["pos"][:, None], case) for x in (s["q"], s["k"])]
    if kind in ("write", "rope_write"):
        key, first = s["k_new"], []
        if kind == "rope_write":
            first = [_rotate_exact(s["q"], s["pos"], case)]
            key = _rotate_exact(key, s["pos"], case).bfloat16()   # the key that is cached
        k, ks = _blocks_exact(s["k"], s["ks"], key, s["slots"])
        v, vs = _blocks_exact(s["v"], s["vs"], s["v_new"], s["slots"])
        return first + [k, v, ks, vs]
    lens, table = s["lens"].tolist(), s["table"].long()

    def rows_of(pool, exponents, b):
        """[Hkv, n, D] values of sequence b."""
        at = torch.arange(lens[b], device="cuda")
        page = table[b, at // P]
        x = pool.view(torch.uint8)[page, :, at % P].view(pool.dtype).float().double()
        e = exponents.view(torch.uint8)[page, :, at % P // _BLOCK].double() - 127
        return (x * torch.exp2(e)[..., None]).transpose(0, 1)

    if kind == "read":
        parts = [[rows_of(s["k"], s["ks"], b), rows_of(s["v"], s["vs"], b)]
                 for b in range(case["S"]) if lens[b]]
        if not parts:
            return [s["k_out"].double(), s["v_out"].double()]
        return [torch.cat([p[i] for p in parts], 1) for i in (0, 1)]
    B, Hq, group = case["B"], case["Hq"], case["Hq"] // case["Hkv"]
    o = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = lens[b]
        if not n:
            continue
        q = s["q"][b].double().view(-1, group, D)
        x = torch.matmul(q, rows_of(s["k"], s["ks"], b).transpose(1, 2).contiguous())
        x = x.reshape(Hq, n) * s["scale"]
        if case["tau"] > 0:
            x = _keep_exact(x, n, case["tau"], case["split"])
        lse[b] = torch.logsumexp(x, -1)
        w = torch.exp(x - lse[b][:, None]).view(-1, group, n)
        o[b] = torch.matmul(w, rows_of(s["v"], s["vs"], b).contiguous()).reshape(Hq, D)
    return [o, lse]


def _keep_exact(x, n, tau, split):
    """Scores [H, n] of one sequence with the tiles that the rule leaves out at -inf; the
    state of a run is the log of the summed weights kept so far."""
    x = x.clone()
    for depth in range(split // _TILE):
        # the tile at this depth below the end of every run
        starts = []
        for run0 in range(0, n, split):
            last = (min(n, run0 + split) - 1) // _TILE
            if last - depth >= run0 // _TILE:
                starts.append((last - depth) * _TILE)
        if not starts:
            break
        at = torch.tensor(starts, device="cuda")
        cols = at[:, None] + torch.arange(_TILE, device="cuda")
        inside = cols < n
        tile = torch.where(inside, x[:, cols.clamp(max=n - 1)], -math.inf)
        state = torch.full(tile.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        if depth:
            after = (at[:, None] + _TILE + torch.arange(_TILE * depth, device="cuda"))
            ends = torch.tensor([min(n, a // split * split + split) for a in starts],
                                device="cuda")
            kept = torch.where(after < ends[:, None], x[:, after.clamp(max=n - 1)], -math.inf)
            state = torch.logsumexp(kept, -1)
        drop = torch.isfinite(state) & (tile.amax(-1) - state < math.log(tau / n))
        tile = torch.where(drop[..., None], -math.inf, tile)
        x[:, cols[inside]] = tile[:, inside]
    return x
