"""The calls of the paged key/value cache whose speed matters: the page tables of a serving
step, new keys and values into pages, pages back to packed rows for a prefill, and the
decode of one token over pages.

Slot of position p of request r: block_table[r][p // P] * P + p % P, P = page size.  Pages are
handed out from a ring of free page numbers, ring[(head + i) % C], and given back at its
end.  A cache holds bf16, or e4m3 with one fp32 scale per KV head (value = e4m3 * scale).
With `own` the calls are the framework's; otherwise the same operators in torch.
"""
import math
import random

import torch

own = False

_TILE = 32           # keys per decision tile of the decode
_E4M3_MAX = 448.0


# ------------------------------------------------------------------ the cases
def listed():
    dec = dict(kind="decode", tau=0.0, split=256, layout="hpd", out="bf16", cache="bf16")
    return [
        # decode: one short sequence, one tensor-parallel rank's heads; latency alone
        dict(dec, name="decode_1x200", B=1, Hq=8, Hkv=2, D=128, P=16, lens="full", n=200),
        # decode: one interactive sequence with every head of a layer, tiles skipped by mass
        dict(dec, name="decode_1x4k", B=1, Hq=32, Hkv=8, D=128, P=64, lens="full", n=4096,
             tau=1e-4, split=128),
        # decode: a serving batch of ragged caches at a coarser tolerance
        dict(dec, name="decode_16x8k_ragged", B=16, Hq=32, Hkv=8, D=128, P=16, lens="uniform",
             n=8192, tau=1e-3, split=256),
        # decode: a larger batch, lengths of every order of magnitude, pages of 8-bit values
        dict(dec, name="decode_64_ragged_e4m3", B=64, Hq=32, Hkv=8, D=128, P=32, lens="log",
             n=16384, cache="e4m3"),
        # decode: multi-head attention of a small model, token-major pages, fp32 output
        dict(dec, name="decode_8x1500_mha_f32", B=8, Hq=16, Hkv=16, D=64, P=48, lens="uniform",
             n=1500, layout="phd", out="f32"),
        # decode: long caches; bandwidth, offsets past 32 bits
        dict(dec, name="decode_16x128k", B=16, Hq=32, Hkv=8, D=128, P=64, lens="full", n=131072),
        # write: the new tokens of a decode step; latency
        dict(kind="write", name="write_64", T=64, Hkv=8, D=128, P=16, slots=16384, cache="bf16",
             layout="hpd", src="tokens", skip=0.0),
        # write: the tokens of long prompts, quantised into token-major pages, some of them
        # padding
        dict(kind="write", name="write_20000_e4m3", T=20000, Hkv=8, D=128, P=32, slots=32768,
             cache="e4m3", layout="phd", src="heads", skip=0.05),
        # read: the cached part of a few prompts of a chunked prefill, 8-bit pages
        dict(kind="read", name="read_4x1000_e4m3", S=4, Hkv=2, D=128, P=16, lens="uniform",
             n=1000, cache="e4m3", layout="hpd"),
        # read: a prefill batch against long cached prefixes
        dict(kind="read", name="read_12x8k", S=12, Hkv=8, D=128, P=64, lens="uniform", n=8192,
             cache="bf16", layout="hpd"),
        # update: a decode step of a running batch, one token each
        dict(kind="update", name="update_decode_64", R=64, P=16, n=4096, mix="decode", tight=0),
        # update: a busy step: prompts admitted, others decoding, finished or cut back, and
        # too few free pages for all of them
        dict(kind="update", name="update_mixed_512", R=512, P=16, n=8192, mix="serve", tight=1),
    ]


def _logsize(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "write", "read", "update"])
    seed = rng.randrange(1 << 30)
    Hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
    P = rng.choice([16, 16, 32, 48, 64, 128, 256])
    common = dict(kind=kind, lseed=seed, P=P)
    cache = rng.choice(["bf16", "bf16", "e4m3"])
    layout = rng.choice(["hpd", "hpd", "phd"])
    if kind == "update":
        return dict(common, R=_logsize(rng, 1, 2048), n=_logsize(rng, 16, 8192),
                    mix=rng.choice(["decode", "serve"]), tight=rng.choice([0, 0, 1]))
    common.update(Hkv=Hkv, D=D, cache=cache, layout=layout)
    if kind == "write":
        T = _logsize(rng, 1, 40000)
        return dict(common, T=T, slots=T + _logsize(rng, 16, 20000),
                    src=rng.choice(["tokens", "heads"]), skip=rng.choice([0.0, 0.05]))
    lens = rng.choice(["full", "uniform", "log"])
    if kind == "read":
        n = _logsize(rng, 1, 16384)
        return dict(common, S=max(1, min(_logsize(rng, 1, 64), 131072 // n)), lens=lens, n=n)
    n = _logsize(rng, 1, 65536)
    return dict(common, B=max(1, min(_logsize(rng, 1, 128), 262144 // n)),
                Hq=Hkv * rng.choice([1, 2, 4, 4, 5, 7, 8, 16]), lens=lens, n=n,
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


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _pool(case, g, num_pages):
    """k, v as [num_pages, Hkv, P, D] views and the scales (None for bf16)."""
    Hkv, P, D = case["Hkv"], case["P"], case["D"]
    e4m3 = case["cache"] == "e4m3"
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    if case["layout"] == "phd":      # token-major pages, K and V of a page side by side
        both = torch.empty((num_pages, 2, P, Hkv, D), dtype=dtype, device="cuda")
        k, v = both[:, 0].permute(0, 2, 1, 3), both[:, 1].permute(0, 2, 1, 3)
        fill = [both]
    else:
        k = torch.empty((num_pages, Hkv, P, D), dtype=dtype, device="cuda")
        v = torch.empty_like(k)
        fill = [k, v]
    for t in fill:
        if not e4m3:
            t.normal_(generator=g)
            continue
        flat, step = t.view(-1), 1 << 27      # e4m3 of normals over a scale of about 1 / 32
        for i in range(0, flat.numel(), step):
            part = flat[i:i + step]
            x = torch.randn(part.numel(), generator=g, device="cuda") * 32
            part.copy_(x.clamp_(-_E4M3_MAX, _E4M3_MAX))
    ks = vs = None
    if e4m3:
        ks = 2.0 ** -5 * (0.75 + 0.5 * torch.rand(Hkv, generator=g, device="cuda"))
        vs = 2.0 ** -5 * (0.75 + 0.5 * torch.rand(Hkv, generator=g, device="cuda"))
    return k, v, ks, vs


def _tables(case, g, lens):
    """Scattered pages for sequences of these lengths: (table [S, W], pages in the pool)."""
    P, W = case["P"], max(1, -(-max(lens) // case["P"]))
    used = [-(-n // P) for n in lens]
    pool = sum(used) + max(1, sum(used) // 8)
    perm = torch.randperm(pool, generator=g, device="cuda").int()
    first = torch.tensor([sum(used[:i]) for i in range(len(used))], device="cuda")
    j = torch.arange(W, device="cuda")
    at = (first[:, None] + j).clamp_(max=pool - 1)
    mine = j < torch.tensor(used, device="cuda")[:, None]
    return torch.where(mine, perm[at], -1).int().contiguous(), pool


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["kind"] == "update":
        return _prepare_update(case, seed, s)
    if case["kind"] == "write":
        pages = -(-case["slots"] // case["P"])
        k, v, ks, vs = _pool(case, g, pages)
        T, Hkv, D = case["T"], case["Hkv"], case["D"]
        if case["src"] == "tokens":           # slices of one [T, 2, Hkv, D] projection
            new = torch.randn((T, 2, Hkv, D), generator=g, device="cuda").bfloat16()
            s["k_new"], s["v_new"] = new[:, 0].transpose(0, 1), new[:, 1].transpose(0, 1)
        else:
            s["k_new"] = torch.randn((Hkv, T, D), generator=g, device="cuda").bfloat16()
            s["v_new"] = torch.randn((Hkv, T, D), generator=g, device="cuda").bfloat16()
        slots = torch.randperm(pages * case["P"], generator=g, device="cuda")[:T].int()
        # the tokens of a prompt lie in runs of whole pages, in the order of the positions
        page = torch.randperm(pages, generator=g, device="cuda")
        t = torch.arange(T, device="cuda")
        runs = (page[t // case["P"]] * case["P"] + t % case["P"]).int()
        slots = runs if T >= 1024 else slots
        skipped = torch.rand(T, generator=g, device="cuda") < case["skip"]
        s["slots"] = torch.where(skipped, -1, slots).int()
    else:
        lens = _lengths(case, case["S"] if case["kind"] == "read" else case["B"])
        s["table"], pages = _tables(case, g, lens)
        k, v, ks, vs = _pool(case, g, pages)
        s["max_len"] = max(max(lens), 1)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        Hkv, D = case["Hkv"], case["D"]
        if case["kind"] == "read":
            cu = [0]
            for n in lens:
                cu.append(cu[-1] + n)
            s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
            s["total"] = max(1, cu[-1])
            s["k_out"] = torch.zeros((Hkv, s["total"], D), dtype=torch.bfloat16, device="cuda")
            s["v_out"] = torch.zeros_like(s["k_out"])
        else:
            # queries that look for the sum of the keys at four places, and noise
            B, Hq = case["B"], case["Hq"]
            q = torch.randn((B, Hq, D), generator=g, device="cuda")
            for _ in range(4):
                at = torch.rand((B, Hq), generator=g, device="cuda")
                at = (at * s["lens"][:, None]).long().clamp_(min=0)
                page = s["table"].gather(1, (at // case["P"]).clamp_(max=s["table"].shape[1] - 1))
                head = torch.arange(Hq, device="cuda") // (Hq // Hkv)
                row = _values(k, ks, (page.long().clamp_(min=0), head.expand(B, Hq),
                                      at % case["P"]))
                q += row * (3.0 if case["tau"] > 0 else 1.0)
            s["q"] = q.bfloat16()
            s["scale"] = D ** -0.5
            o_type = torch.float32 if case["out"] == "f32" else torch.bfloat16
            s["o"] = torch.empty((B, Hq, D), dtype=o_type, device="cuda")
            s["lse"] = torch.empty((B, Hq), dtype=torch.float32, device="cuda")
    s.update(k=k, v=v, ks=ks, vs=vs)
    if own:      # what a serving program makes once: the handle of its cache, a workspace
        import paper_2609_32712_amd as mala
        s["cache"] = mala.PagedCache(k, v, ks, vs)
        if case["kind"] == "decode":
            need = mala.mala_paged_decode_workspace_size(case["B"], case["Hq"], case["Hkv"],
                                                         case["D"], s["max_len"], case["split"])
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


def _values(pool, scale, index):
    """fp32 values of pool[page, head, row] for index tensors of one shape."""
    page, head, row = index
    raw = pool.view(torch.uint8)[page, head, row].view(pool.dtype) if scale is not None else \
        pool[page, head, row]
    x = raw.float()
    return x if scale is None else x * scale[head][..., None]


def _update_plan(case):
    """Old and new lengths of the requests of a step, from the case alone."""
    rng, R, n = random.Random(case.get("lseed", 1)), case["R"], case["n"]
    old, new = [], []
    for i in range(R):
        have = rng.randint(1, max(1, n - 1))
        what = 0.0 if case["mix"] == "decode" else rng.random()
        if what < 0.7:
            a, b = have, have + 1                       # decodes one token
        elif what < 0.8:
            a, b = 0, have                              # a prompt is admitted
        elif what < 0.86:
            a, b = have, min(n, have + rng.randint(1, 512))   # the next chunk of a prompt
        elif what < 0.94:
            a, b = have, 0                              # finished
        elif what < 0.97:
            a, b = have, max(0, have - rng.randint(1, 64))    # rejected tokens taken back
        else:
            a, b = 0, 0                                 # an idle row
        old.append(a)
        new.append(b)
    return old, new


def _update_sizes(case):
    old, new = _update_plan(case)
    P = case["P"]
    have, want = [-(-a // P) for a in old], [-(-b // P) for b in new]
    need = sum(max(0, w - h) for h, w in zip(have, want))
    free = need * 6 // 10 if case["tight"] else need + 8
    tokens = sum(max(0, b - a) for a, b in zip(old, new))
    return old, new, have, want, need, free, tokens


def _prepare_update(case, seed, s):
    old, new, have, want, need, free, tokens = _update_sizes(case)
    g = _gen(seed)
    W = -(-case["n"] // case["P"]) + 1
    pool = sum(have) + free
    perm = torch.randperm(pool, generator=g, device="cuda").int()
    h = torch.tensor(have, device="cuda")
    first = h.cumsum(0) - h
    j = torch.arange(W, device="cuda")
    at = (first[:, None] + j).clamp_(max=pool - 1)
    s["table"] = torch.where(j < h[:, None], perm[at], -1).int().contiguous()
    head = int(torch.randint(pool, (1,), generator=g, device="cuda"))
    ring = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(free, device="cuda")) % pool] = perm[sum(have):]
    s["ring"], s["pool"] = ring, pool
    s["state"] = torch.tensor([head, free, 0, 0], dtype=torch.int32, device="cuda")
    s["lens"] = torch.tensor(old, dtype=torch.int32, device="cuda")
    s["new_lens"] = torch.tensor(new, dtype=torch.int32, device="cuda")
    cap = -(-tokens // 64) * 64 + 64         # a captured step pads its tokens
    R = case["R"]
    i32 = dict(dtype=torch.int32, device="cuda")
    s["lens_out"], s["cu"] = torch.empty(R, **i32), torch.empty(R + 1, **i32)
    s["slots"], s["positions"] = torch.empty(cap, **i32), torch.empty(cap, **i32)
    s["state_out"] = torch.empty(4, **i32)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"update": _own_update, "write": _own_write, "read": _own_read,
                "decode": _own_decode}[kind](s)
    return {"update": _plain_update, "write": _plain_write, "read": _plain_read,
            "decode": _plain_decode}[kind](s)


def _own_update(s):
    import paper_2609_32712_amd as mala
    mala.mala_paged_update(s["lens"], s["new_lens"], s["table"], s["ring"], s["state"],
                           s["lens_out"], s["cu"], s["slots"], s["positions"], s["state_out"],
                           s["case"]["P"], s["pool"])
    return [s["table"], s["ring"], s["lens_out"], s["cu"], s["slots"], s["positions"],
            s["state_out"]]


def _own_write(s):
    import paper_2609_32712_amd as mala
    mala.mala_paged_write(s["k_new"], s["v_new"], s["slots"], s["cache"])
    return [s["k"], s["v"]]


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


def _plain_update(s):
    case, table, ring = s["case"], s["table"], s["ring"]
    P, pool, (R, W), C = case["P"], s["pool"], table.shape, ring.numel()
    old, new = s["lens"].long().clamp(0, W * P), s["new_lens"].long().clamp(0, W * P)
    head, count = s["state"][0].long(), s["state"][1].long()
    have, want = (old + P - 1) // P, (new + P - 1) // P
    need, back = (want - have).clamp(min=0), (have - want).clamp(min=0)
    end = need.cumsum(0)
    granted = (need == 0) | (end <= count)
    taken = torch.where(granted, need, 0).sum()
    lens_out = torch.where(granted, new, old).int()
    cu = torch.nn.functional.pad((new - old).clamp(min=0).cumsum(0), (1, 0))
    t = torch.arange(s["slots"].numel(), device="cuda")
    r = torch.searchsorted(cu[1:], t, right=True).clamp(max=R - 1)
    pos, live = old[r] + t - cu[r], t < cu[-1]
    page = (pos // P).clamp(max=W - 1)
    fresh = ring[(head + (end - need)[r] + page - have[r]) % C]
    number = torch.where(page >= have[r], fresh, table[r, page]).long()
    good = live & granted[r] & (number >= 0) & (number < pool)
    slots = torch.where(good, number * P + pos % P, -1).int()
    positions = torch.where(live, pos, 0).int()
    # table rows and the ring's end (entry C of the longer copy takes what is not given back)
    j = torch.arange(W, device="cuda")
    place = (back.cumsum(0) - back)[:, None] + j - want[:, None]
    given = (j >= want[:, None]) & (j < have[:, None])
    longer = torch.nn.functional.pad(ring, (0, 1))
    longer.scatter_(0, torch.where(given, (head + count + place) % C, C).view(-1), table.view(-1))
    added = (j >= have[:, None]) & (j < want[:, None]) & granted[:, None]
    popped = ring[(head + (end - need)[:, None] + j - have[:, None]) % C]
    table.copy_(torch.where(added, popped, table))
    ring.copy_(longer[:C])
    state = torch.stack([(head + taken) % C, count - taken + back.sum(), (~granted).sum(),
                         cu[-1]]).int()
    return [table, ring, lens_out, cu.int(), slots, positions, state]


def _plain_write(s):
    P = s["case"]["P"]
    pages = s["k"].shape[0]
    # tokens without a slot go to slot 0 of one page more than the cache has
    slot = torch.where((s["slots"] >= 0) & (s["slots"] < pages * P), s["slots"], pages * P).long()
    for pool, scale, new in ((s["k"], s["ks"], s["k_new"]), (s["v"], s["vs"], s["v_new"])):
        x = new.transpose(0, 1).float()
        if scale is not None:
            x = (x / scale[:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(pool.dtype)
            pool, x = pool.view(torch.uint8), x.view(torch.uint8)
        else:
            x = x.to(pool.dtype)
        longer = torch.cat([pool, pool[:1]])
        longer[slot // P, :, slot % P] = x
        pool.copy_(longer[:pages])
    return [s["k"], s["v"]]


def _gathered(pool, table, width):
    """[S, Hkv, width * P, D] fp32 (unscaled) rows of the first `width` pages of each table row."""
    raw = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
    x = raw[table[:, :width].long().clamp(min=0)].permute(0, 2, 1, 3, 4)
    S, H, W, P, D = x.shape
    return x.reshape(S, H, W * P, D).view(pool.dtype).float()


def _plain_read(s):
    P, lens = s["case"]["P"], s["lens"]
    width = -(-s["max_len"] // P)
    t = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(s["cu"][1:], t.int(), right=True).clamp(max=lens.numel() - 1)
    pos = t - s["cu"][seq].long()
    page = s["table"][seq, (pos // P).clamp(max=width - 1)].long().clamp(min=0)
    for pool, scale, out in ((s["k"], s["ks"], s["k_out"]), (s["v"], s["vs"], s["v_out"])):
        raw = pool.view(torch.uint8) if scale is not None else pool
        x = raw[page, :, pos % P].view(pool.dtype).float()
        if scale is not None:
            x = x * scale[:, None]
        out.copy_(torch.where((t < s["cu"][-1])[:, None], x.transpose(0, 1), out))
    return [s["k_out"], s["v_out"]]


def _plain_decode(s):
    case, table, lens = s["case"], s["table"], s["lens"]
    B, Hq, Hkv, D, P = case["B"], case["Hq"], case["Hkv"], case["D"], case["P"]
    width = -(-s["max_len"] // P)
    N = width * P
    k = _gathered(s["k"], table, width)
    score = torch.matmul(s["q"].float().view(B, Hkv, Hq // Hkv, D), k.transpose(2, 3)) * s["scale"]
    del k
    if s["ks"] is not None:
        score = score * s["ks"][:, None, None]
    pos = torch.arange(N, device="cuda")
    seen = (pos < lens[:, None]) & (table[:, :width] >= 0).repeat_interleave(P, 1)
    score = score.masked_fill(~seen[:, None, None], -math.inf).view(B, Hq, N)
    if case["tau"] > 0:
        score = score.masked_fill(~_retained(score, lens, case["tau"], case["split"]), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    v = _gathered(s["v"], table, width)
    o = torch.matmul(p.view(B, Hkv, Hq // Hkv, N), v).view(B, Hq, D)
    if s["vs"] is not None:
        o = o * s["vs"].repeat_interleave(Hq // Hkv)[:, None]
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
    if case["kind"] == "update":
        old, new, have, want, need, free, tokens = _update_sizes(case)
        got = min(need, free)
        back = sum(max(0, h - w) for h, w in zip(have, want))
        cap = -(-tokens // 64) * 64 + 64
        return dict(bytes=4 * (4 * case["R"] + 2 * got + 2 * back + 2 * cap), flops=0)
    e = 1 if case["cache"] == "e4m3" else 2
    row = 2 * case["Hkv"] * case["D"]        # values of K and V of a token
    if case["kind"] == "write":
        return dict(bytes=case["T"] * (row * (2 + e) + 4), flops=0)
    lens = _lengths(case, case["S"] if case["kind"] == "read" else case["B"])
    pages = sum(-(-n // case["P"]) for n in lens)
    if case["kind"] == "read":
        return dict(bytes=sum(lens) * row * (2 + e) + 4 * pages, flops=0)
    heads = case["B"] * case["Hq"]
    ends = heads * (case["D"] * (2 + (4 if case["out"] == "f32" else 2)) + 4)
    return dict(bytes=sum(lens) * row * e + 4 * pages + ends,
                flops=4 * sum(lens) * case["Hq"] * case["D"])


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["kind"] == "update":
        return None                          # whole numbers only
    s = prepare(case, seed)
    P, D = case["P"], case["D"]
    one = torch.ones(case["Hkv"], dtype=torch.float64, device="cuda")
    ks, vs = (one if x is None else x.double() for x in (s["ks"], s["vs"]))
    if case["kind"] == "write":
        result = []
        hit = ((s["slots"] >= 0) & (s["slots"] < s["k"].shape[0] * P)).nonzero().view(-1)
        slot = s["slots"][hit].long()
        for pool, scale, new in ((s["k"], ks, s["k_new"]), (s["v"], vs, s["v_new"])):
            rows = pool.float().double()
            x = new.double()[:, hit] / scale[:, None, None]
            if pool.dtype == torch.float8_e4m3fn:
                x = x.clamp(-_E4M3_MAX, _E4M3_MAX)
            for h in range(case["Hkv"]):
                rows[slot // P, h, slot % P] = x[h]
            result.append(rows)
        return result
    lens, table = s["lens"].tolist(), s["table"].long()

    def rows_of(pool, scale, b):
        """[Hkv, n, D] values of sequence b."""
        at = torch.arange(lens[b], device="cuda")
        raw = pool if pool.dtype == torch.bfloat16 else pool.view(torch.uint8)
        x = raw[table[b, at // P], :, at % P].view(pool.dtype).float().double()
        return x.transpose(0, 1) * scale[:, None, None]

    if case["kind"] == "read":
        parts = [[rows_of(s["k"], ks, b), rows_of(s["v"], vs, b)]
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
        x = torch.matmul(q, rows_of(s["k"], ks, b).transpose(1, 2).contiguous())
        x = x.reshape(Hq, n) * s["scale"]
        if case["tau"] > 0:
            x = _keep_exact(x, n, case["tau"], case["split"])
        lse[b] = torch.logsumexp(x, -1)
        w = torch.exp(x - lse[b][:, None]).view(-1, group, n)
        o[b] = torch.matmul(w, rows_of(s["v"], vs, b).contiguous()).reshape(Hq, D)
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
