"""Cases, plain forms and 64-bit definitions of the paged-cache operators.

Four operators that a serving program uses in this order, all on [B][H][n][d] tensors:

  rotary   y = m * (x rotated by the angles  position * inv_freq)   (the transposed rotation is its gradient)
  append   rotates a chunk's queries and keys, writes keys and values into the pages of a cache
  attend   attention of the chunk over its cache pages, log-sum-exp, and the decayed score of every cached token
           S <- alpha^len S + sum_i alpha^(len-1-i) P_i    (summed over the query heads of a key/value head)
  evict    brings a sequence back to its budget: the newest `recent` positions stay, of the others the best by
           (score, position); in place, or into other pages when the old ones are shared

A cache page holds ``ps`` slots of every key/value head: k_pages, v_pages [pages][H][ps][d], scores and positions
[pages][H][ps]; page_table [B][max_pages].  ``past`` [B] slots are in use before the chunk, ``start`` [B] tokens were seen.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # a whole prompt batch's queries before a dense prefill: the largest tensor of the workloads
        dict(name="rotary_prompt", op="rotary", B=32, H=40, n=4096, d=128, dtype="bf16", r=128, interleaved=False, scaling="none", start=0,
             ragged=False, transpose=False),
        # gradient of a partly rotated head at far positions, neighbouring pairs, odd length, 32-bit storage
        dict(name="rotary_grad_far", op="rotary", B=4, H=12, n=1023, d=64, dtype="fp32", r=32, interleaved=True, scaling="ramp", start=900001,
             ragged=True, transpose=True),
        # one token of every sequence enters the cache: latency
        dict(name="append_token", op="append", B=32, H=40, G=1, d=128, dtype="bf16", ps=64, past=511, c=1, ragged=True, r=128,
             interleaved=False, scaling="none"),
        # a ragged batch of prompt chunks behind a cached prefix, grouped heads
        dict(name="append_chunk", op="append", B=8, H=8, G=4, d=128, dtype="fp16", ps=32, past=1000, c=2047, ragged=True, r=128,
             interleaved=False, scaling="bands"),
        # one token over a pruned cache of 205 slots: the smallest call
        dict(name="attend_token_small", op="attend", B=1, H=32, G=1, d=128, dtype="bf16", ps=16, past=204, c=1, ragged=False, alpha=0.3),
        # one token of every sequence over its full, ragged cache: bound by the cache's bytes
        dict(name="attend_token_full", op="attend", B=32, H=40, G=1, d=128, dtype="bf16", ps=64, past=4095, c=1, ragged=True, alpha=0.5),
        # four drafted tokens over two long caches, grouped heads
        dict(name="attend_draft_long", op="attend", B=2, H=8, G=4, d=128, dtype="fp16", ps=64, past=32700, c=4, ragged=False, alpha=0.9),
        # a chunk of a long prompt: bound by the matrix products
        dict(name="attend_chunk_long", op="attend", B=1, H=32, G=1, d=128, dtype="bf16", ps=128, past=30720, c=2048, ragged=False, alpha=0.9),
        # whole prompts in one chunk, grouped heads, plain accumulated scores
        dict(name="attend_prompt_group", op="attend", B=8, H=8, G=4, d=128, dtype="fp16", ps=64, past=0, c=2048, ragged=True, alpha=1.0),
        # a small 32-bit prompt of odd length, heads of 64
        dict(name="attend_prompt_fp32", op="attend", B=2, H=4, G=1, d=64, dtype="fp32", ps=16, past=0, c=129, ragged=False, alpha=0.5),
        # the end of the prompt: 4096 tokens a head to 512, into fresh pages (the prompt's pages may be shared)
        dict(name="evict_prompt", op="evict", B=32, H=40, G=1, d=128, dtype="bf16", ps=64, past=4095, c=1, budget=512, recent=256, fresh=True),
        # the cache's part of a generation step: four tokens enter a full cache, four leave it, in place
        dict(name="evict_step", op="evict", B=8, H=32, G=1, d=128, dtype="fp16", ps=32, past=2048, c=4, budget=2048, recent=1024, fresh=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "attend", "attend", "evict"])
    dtype, d, ps = rng.choice(["fp32", "bf16", "bf16", "fp16"]), rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    r = rng.choice([d, d, d // 2, 24, 16])
    angles = dict(r=r, interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "ntk", "bands", "ramp"]))
    ragged = rng.random() < 0.5
    if op == "rotary":
        B, H, n = _log(rng, 1, 32), _log(rng, 1, 40), _log(rng, 1, 4096)
        return dict(op=op, B=B, H=H, n=n, d=d, dtype=dtype, **angles, start=_log(rng, 1, 1000000), ragged=ragged, transpose=rng.random() < 0.5)
    H, G = _log(rng, 1, 32), rng.choice([1, 1, 2, 4, 5, 8])
    if op == "append":
        B, c = _log(rng, 1, 32), _log(rng, 1, 2048)
        B, H = (min(B, 8), min(H, 8)) if c > 256 else (B, H)
        return dict(op=op, B=B, H=H, G=G, d=d, dtype=dtype, ps=ps, past=_log(rng, 1, 2000), c=c, ragged=ragged, **angles)
    if op == "evict":
        B, past = _log(rng, 1, 16), _log(rng, 64, 8192)
        c = rng.choice([1, 3, 17])
        fresh = rng.random() < 0.5
        budget = max(40, past // rng.choice([2, 5, 8])) if fresh else past
        return dict(op=op, B=B, H=min(H, max(1, (1 << 20) // (B * past))), G=1, d=d, dtype=dtype, ps=ps, past=past, c=c, budget=budget,
                    recent=rng.choice([budget // 2, 32]), fresh=fresh)
    c, past = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 2048)]), rng.choice([0, _log(rng, 1, 32768), _log(rng, 1, 32768)])
    B = _log(rng, 1, 32)
    dense = 2 ** 24 if dtype == "fp32" else 2 ** 30               # logits of the call: fp32 storage is for small models
    rows = 2 ** 21 if dtype == "fp32" else 2 ** 22                # cached rows of the call
    while B * H * G * c * (past + c) > dense or B * H * (past + c) > rows:
        if max(B, H) > 1:
            B, H = (B // 2, H) if B >= H else (B, H // 2)
        elif c > 1:
            c = c // 2
        else:
            past = past // 2
    return dict(op=op, B=B, H=H, G=G, d=d, dtype=dtype, ps=ps, past=past, c=c, ragged=ragged, alpha=rng.choice([0.0, 0.3, 0.5, 0.9, 1.0]))


# ---- what the cases say, as numbers -------------------------------------------------------------------------------

def _spread(most, B, ragged, shift):
    """Lengths of the batch: all `most`, or spread over 0 .. most (the first one is the longest)."""
    return [int(most * (1.0 - 0.95 * ((b * 0.6180339887 + shift * b) % 1.0))) if ragged else most for b in range(B)]


def _lens(c):
    n = c["n"] if c["op"] == "rotary" else c["c"]
    return _spread(n, c["B"], c.get("ragged", False) and n > 1, 0.37)


def _past(c):
    return _spread(c["past"], c["B"], c.get("ragged", False), 0.0)


def _rope(c):
    """What the rotary plan is made of."""
    scaling = c["scaling"]
    return dict(rotary_dim=c["r"], theta=10000.0, interleaved=c["interleaved"], scaling=scaling, factor=1.0 if scaling == "none" else 8.0,
                original_length=4096, low=1.0, high=32.0 if scaling == "ramp" else 4.0)


def _inv_freq(c):
    """Frequencies (64 bits) and magnitude of the rotation."""
    p = _rope(c)
    r, theta, factor, L = p["rotary_dim"], p["theta"], p["factor"], p["original_length"]
    i = np.arange(r // 2, dtype=np.float64)
    if p["scaling"] == "ntk":
        theta = theta * factor ** (r / (r - 2.0))
    f = theta ** (-2.0 * i / r)
    if p["scaling"] == "linear":
        f = f / factor
    if p["scaling"] == "bands":
        wave = 2.0 * math.pi / f
        t = np.clip((L / wave - p["low"]) / (p["high"] - p["low"]), 0.0, 1.0)
        f = (1.0 - t) * f / factor + t * f
    if p["scaling"] == "ramp":
        at = [r * math.log(L / (2.0 * math.pi * beta)) / (2.0 * math.log(theta)) for beta in (p["high"], p["low"])]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        t = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        f = t * f / factor + (1.0 - t) * f
    return f, (0.1 * math.log(factor) + 1.0 if p["scaling"] == "ramp" else 1.0)


def work(c):
    e, d = BYTES[c["dtype"]], c["d"]
    if c["op"] == "rotary":
        rows = c["H"] * sum(_lens(c))
        return {"bytes": 2 * rows * d * e, "flops": 3 * rows * c["r"]}
    H, G, lens, past = c["H"], c["G"], _lens(c), _past(c)
    if c["op"] == "append":
        rows = H * sum(lens)
        return {"bytes": rows * ((4 + 2 * G) * d * e + 8), "flops": 3 * rows * (G + 1) * c["r"]}
    if c["op"] == "attend":
        seen = sum(H * (p + n) for p, n in zip(past, lens) if n)
        pairs = sum(H * G * (n * p + n * (n + 1) // 2) for p, n in zip(past, lens))
        rows = sum(H * G * n for n in lens)
        return {"bytes": seen * (2 * d * e + 8) + rows * (2 * d * e + 4), "flops": 4 * d * pairs}
    units, n, M = c["B"] * H, c["past"] + c["c"], min(c["budget"], c["past"] + c["c"])
    moved = M if c["fresh"] else n - M                             # rows that have to change their place
    enter = 0 if c["fresh"] else c["c"] * (4 * d * e + 8)           # the appended tokens of a step
    return {"bytes": units * (8 * n + moved * (4 * d * e + 8) + enter), "flops": units * n}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _normal(gen, shape, dtype):
    return torch.randn(shape, dtype=dtype if dtype != torch.float32 else None, device="cuda", generator=gen)


def _cache(c, gen, slots):
    """Pool, page table (pages in no order) and lengths; every slot of the pool holds something."""
    B, H, d, ps, dt = c["B"], c["H"], c["d"], c["ps"], DTYPES[c["dtype"]]
    mp = -(-slots // ps)
    extra = -(-c["budget"] // ps) if c.get("fresh") else 0
    pages = B * (mp + extra) + 1
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    s = dict(k_pages=_normal(gen, (pages, H, ps, d), dt), v_pages=_normal(gen, (pages, H, ps, d), dt),
             page_table=order[: B * mp].view(B, mp).contiguous(), dst_table=order[B * mp: B * (mp + extra)].view(B, extra).contiguous() if extra else None,
             past=_int(_past(c)), start=_int(_past(c)), lens=_int(_lens(c)))
    s["k_pages"][s["page_table"][:, 0].long(), :, 0] *= 4            # the first token of a sequence draws attention
    # scores: a few heavy tokens, many light ones, and many that are equal
    u = torch.rand((pages, H, ps), device="cuda", generator=gen)
    s["scores"] = torch.where(u < 0.3, torch.zeros_like(u), u ** 8)
    s["positions"] = torch.full((pages, H, ps), -1, dtype=torch.int32, device="cuda")
    slot = torch.arange(mp * ps, dtype=torch.int32, device="cuda").view(1, mp, 1, ps).expand(B, mp, H, ps)
    s["positions"][s["page_table"].view(-1).long()] = slot.reshape(B * mp, H, ps)
    return s


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, d = DTYPES[c["dtype"]], c["d"]
    if c["op"] == "rotary":
        x = _normal(gen, (c["B"], c["H"], c["n"], d), dt)
        s = dict(x=x, out=torch.zeros_like(x), lens=_int(_lens(c)), start=_int([c["start"] + 17 * b for b in range(c["B"])]))
    else:
        B, H, G, n = c["B"], c["H"], c["G"], c["c"]
        s = _cache(c, gen, c["past"] + n)
        if c["op"] != "attend" and not c.get("fresh"):
            s["k"], s["v"] = _normal(gen, (B, H, n, d), dt), _normal(gen, (B, H, n, d), dt)
        if c["op"] in ("append", "attend"):
            s["q"] = _normal(gen, (B, H * G, n, d), dt)
            s["out"] = torch.zeros_like(s["q"])
        if c["op"] == "append":
            s["start"] = s["start"] + 7
        if c["op"] == "attend":
            s["lse"] = torch.zeros((B, H * G, n), dtype=torch.float32, device="cuda")
        if c["op"] == "evict":
            s["past_out"], s["start_out"] = (torch.empty_like(s["past"]), torch.empty_like(s["past"])) if c["fresh"] else (s["past"], s["start"])
    s["case"] = c
    if "r" in c:
        s["inv_freq"], s["magnitude"] = _inv_freq(c)
        s["inv_freq"] = torch.from_numpy(s["inv_freq"]).cuda()
    if own:                                                        # the handles that a program keeps
        from paper_2407_20485_b200 import binding as a2sf
        if "r" in c:
            s["plan"] = a2sf.a2sf_rotary_plan_init(**_rope(c))
        if c["op"] != "rotary":
            s["cache"] = a2sf.PagedCache(c["B"], c["H"], d, dt, c["ps"], s["k_pages"].shape[0], s["page_table"].shape[1], group=c["G"],
                                         **{k: s[k] for k in ("k_pages", "v_pages", "scores", "positions", "page_table", "past", "start")})
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _rotated(x, pos, inv_freq, magnitude, interleaved, transpose):
    """x [B][H][n][d] rotated by pos [B][n]: angles in 64 bits, arithmetic in 32, one rounding."""
    half = inv_freq.numel()
    ang = pos[:, None, :, None].double() * inv_freq
    cos, sin = (torch.cos(ang) * magnitude).float(), (torch.sin(ang) * magnitude).float()
    if transpose:
        sin = -sin
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    x1, x2 = x[..., a].float(), x[..., b].float()
    y = x.clone()
    y[..., a] = (x1 * cos - x2 * sin).to(x.dtype)
    y[..., b] = (x2 * cos + x1 * sin).to(x.dtype)
    return y


def _rotary(s):
    c, x = s["case"], s["x"]
    t = torch.arange(x.shape[2], device="cuda")
    y = _rotated(x, s["start"][:, None] + t, s["inv_freq"], s["magnitude"], c["interleaved"], c["transpose"])
    return {"out": torch.where((t < s["lens"][:, None])[:, None, :, None], y, s["out"])}


def _place(s, slot):
    """Page and slot in the page of cache slots [B][n]."""
    ps = s["k_pages"].shape[2]
    return torch.gather(s["page_table"].long(), 1, slot // ps), slot % ps


def _append(s, k, q=None):
    """Writes k (already rotated) and v where they belong; scores start at zero."""
    n = k.shape[2]
    t = torch.arange(n, device="cuda")
    b, i = torch.nonzero((t < s["lens"][:, None]), as_tuple=True)
    slot = s["past"].long()[:, None] + t
    page, off = _place(s, torch.minimum(slot, torch.full_like(slot, s["page_table"].shape[1] * s["k_pages"].shape[2] - 1)))
    page, off = page[b, i], off[b, i]
    s["k_pages"][page, :, off] = k[b, :, i]
    s["v_pages"][page, :, off] = s["v"][b, :, i]
    s["scores"][page, :, off] = 0.0
    s["positions"][page, :, off] = (s["start"][b] + i.to(torch.int32))[:, None].expand(-1, k.shape[1])


def _append_rotated(s):
    c = s["case"]
    t = torch.arange(s["k"].shape[2], device="cuda")
    pos = s["start"][:, None] + t
    k, q = (_rotated(x, pos, s["inv_freq"], s["magnitude"], c["interleaved"], False) for x in (s["k"], s["q"]))
    _append(s, k)
    q = torch.where((t < s["lens"][:, None])[:, None, :, None], q, s["out"])
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"], "scores": s["scores"], "positions": s["positions"]}


def _attend(s):
    c = s["case"]
    B, H, G, d, n = c["B"], c["H"], c["G"], c["d"], c["c"]
    table = s["page_table"].long()
    kv = [p[table].transpose(1, 2).reshape(B, H, -1, d).float() for p in (s["k_pages"], s["v_pages"])]
    L = kv[0].shape[2]
    q = s["q"].float().view(B, H, G * n, d)
    t, j = torch.arange(n, device="cuda"), torch.arange(L, device="cuda")
    past, lens = s["past"].long()[:, None], s["lens"].long()[:, None]
    live = t < lens                                                   # [B][n]
    seen = (j <= (past + t)[:, :, None]) & live[:, :, None]           # [B][n][L]
    x = torch.matmul(q, kv[0].transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, H, G, n, L)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min_(-3.0e38)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    x = x.div_(total.clamp_min(1e-38))
    out = torch.matmul(x.view(B, H, G * n, L), kv[1]).view(B, H * G, n, d).to(s["out"].dtype)
    lse = (m + torch.log(total)).view(B, H * G, n)
    age = (lens - 1 - t).clamp_min(0)
    weight = torch.where(live, torch.pow(torch.full_like(age, c["alpha"], dtype=torch.float64), age), torch.zeros((), dtype=torch.float64, device="cuda")).float()
    gain = torch.matmul(weight.repeat(1, G)[:, None, None, :], x.view(B, H, G * n, L)).view(B, H, -1, c["ps"])
    decay = torch.pow(torch.full_like(lens, c["alpha"], dtype=torch.float64), lens).float()[:, :, None, None]
    b, page = torch.nonzero((torch.arange(table.shape[1], device="cuda") * c["ps"] < past + lens) & (lens > 0), as_tuple=True)
    here = (j < past + lens).view(B, 1, -1, c["ps"]).transpose(1, 2)    # slots in use
    old = s["scores"][table]
    new = torch.where(here, old * decay + gain.transpose(1, 2), old)
    s["scores"][table[b, page]] = new[b, page]
    mask = live[:, None, :]
    return {"out": torch.where(mask[..., None], out, s["out"]), "lse": torch.where(mask, lse, s["lse"]), "scores": s["scores"]}


def _evict(s):
    c = s["case"]
    B, H, d, ps, M = c["B"], c["H"], c["d"], c["ps"], c["budget"]
    if not c["fresh"]:
        _append(s, s["k"])
    table = s["page_table"].long()
    sc, pos = (s[x][table].transpose(1, 2).reshape(B, H, -1) for x in ("scores", "positions"))
    L = sc.shape[2]
    j = torch.arange(L, device="cuda")
    n = (s["past"] + s["lens"]).long()
    m = torch.clamp(n, max=M)
    newest = (s["start"] + s["lens"] - c["recent"])[:, None, None]
    bits = sc.contiguous().view(torch.int32).long()                    # scores are not negative: their bits are in their order
    key = torch.where(pos >= newest, torch.full_like(bits, 2 ** 62), bits * 2 ** 31 + pos)
    key = torch.where(j < n[:, None, None], key, torch.full_like(key, -1))
    order = torch.argsort(key, dim=2, stable=True)
    rank = torch.empty_like(order).scatter_(2, order, j.expand_as(order).contiguous())
    keep = rank >= L - m[:, None, None]
    if c["fresh"]:
        src = torch.nonzero(keep, as_tuple=True)
        to = (torch.cumsum(keep, 2) - 1)[src]
        to_page = s["dst_table"].long()[src[0], to // ps]
    else:
        src = torch.nonzero(keep & (j >= m[:, None, None]), as_tuple=True)
        to = torch.nonzero(~keep & (j < m[:, None, None]), as_tuple=True)[2]
        to_page = table[src[0], to // ps]
    page, h = table[src[0], src[2] // ps], src[1]
    for x in ("k_pages", "v_pages", "scores", "positions"):
        s[x][to_page, h, to % ps] = s[x][page, h, src[2] % ps]
    start = s["start"] + s["lens"]
    s["past_out"].copy_(m)
    s["start_out"].copy_(start)
    return {x: s[x] for x in ("k_pages", "v_pages", "scores", "positions", "past_out", "start_out")}


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"rotary": _rotary, "append": _append_rotated, "attend": _attend, "evict": _evict}[c["op"]](s)
    if c["op"] == "rotary":
        from paper_2407_20485_b200 import binding as a2sf
        return {"out": a2sf.a2sf_rotary(s["plan"], s["x"], out=s["out"], start=s["start"], lens=s["lens"], transpose=c["transpose"])}
    cache = s["cache"]
    pool = {x: s[x] for x in ("k_pages", "v_pages", "scores", "positions")}
    if c["op"] == "append":
        q = cache.a2sf_paged_append(s["k"], s["v"], lens=s["lens"], q=s["q"], q_out=s["out"], rotary=s["plan"])
        return {"q": q, **pool}
    if c["op"] == "attend":
        out, lse = cache.a2sf_paged_attend(s["q"], c["alpha"], lens=s["lens"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse, "scores": s["scores"]}
    if not c["fresh"]:
        cache.a2sf_paged_append(s["k"], s["v"], lens=s["lens"])
    cache.a2sf_paged_evict(c["budget"], c["recent"], c["c"], lens=s["lens"], dst_table=s["dst_table"], past_out=s["past_out"], start_out=s["start_out"])
    return {**pool, "past_out": s["past_out"], "start_out": s["start_out"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def _turn(x, positions, c):
    """x [H][n][d] in 64 bits, pair by pair as complex numbers."""
    f, m = _inv_freq(c)
    h = len(f)
    z = torch.from_numpy(f).cuda()[None, :] * positions.double()[:, None]
    z = torch.polar(torch.full_like(z, m), -z if c.get("transpose") else z)
    y = x.clone()
    if c["interleaved"]:
        y[..., : 2 * h] = torch.view_as_real(torch.view_as_complex(x[..., : 2 * h].reshape(*x.shape[:-1], h, 2).contiguous()) * z).flatten(-2)
    else:
        w = torch.complex(x[..., :h].contiguous(), x[..., h: 2 * h].contiguous()) * z
        y[..., :h], y[..., h: 2 * h] = w.real, w.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    lens = _lens(c)
    if c["op"] == "rotary":
        out = s["out"].double()
        for b, n in enumerate(lens):
            out[b, :, :n] = _turn(s["x"][b, :, :n].double(), torch.arange(n, device="cuda") + int(s["start"][b]), c)
        return {"out": out}
    past, ps, table = _past(c), c["ps"], s["page_table"].long()
    if c["op"] == "attend":
        G, H = c["G"], c["H"]
        out, lse, scores = s["out"].double(), s["lse"].double(), s["scores"].double()
        for b, n in enumerate(lens):
            if not n:
                continue
            L = past[b] + n
            slots = torch.arange(L, device="cuda")
            pg, off = table[b, slots // ps], slots % ps
            i = torch.arange(n, device="cuda")
            hidden = slots[None, :] > past[b] + i[:, None]
            w = torch.tensor([float(c["alpha"]) ** (n - 1 - x) for x in range(n)], dtype=torch.float64, device="cuda")
            for h in range(H):
                K, V = s["k_pages"][pg, h, off].double(), s["v_pages"][pg, h, off].double()
                gain = torch.zeros(L, dtype=torch.float64, device="cuda")
                for g in range(h * G, h * G + G):
                    x = (s["q"][b, g, :n].double() @ K.T) / math.sqrt(c["d"])
                    x[hidden] = -math.inf
                    z = torch.logsumexp(x, 1)
                    P = torch.exp(x - z[:, None])
                    out[b, g, :n], lse[b, g, :n] = P @ V, z
                    gain += w @ P
                scores[pg, h, off] = scores[pg, h, off] * float(c["alpha"]) ** n + gain
        return {"out": out, "lse": lse, "scores": scores}
    pool = {x: s[x].double() if s[x].is_floating_point() else s[x] for x in ("k_pages", "v_pages", "scores", "positions")}
    if c["op"] == "append" or not c["fresh"]:
        q = s["out"].double() if c["op"] == "append" else None
        for b, n in enumerate(lens):
            if not n:
                continue
            at = torch.arange(n, device="cuda")
            pg, off = table[b, (past[b] + at) // ps], (past[b] + at) % ps
            k, pos = s["k"][b, :, :n].double(), at + int(s["start"][b])
            if c["op"] == "append":
                k = _turn(k, pos, c)
                q[b, :, :n] = _turn(s["q"][b, :, :n].double(), pos, c)
            pool["k_pages"][pg, :, off] = k.transpose(0, 1)
            pool["v_pages"][pg, :, off] = s["v"][b, :, :n].double().transpose(0, 1)
            pool["scores"][pg, :, off] = 0.0
            pool["positions"][pg, :, off] = pos.to(torch.int32)[:, None]
        if c["op"] == "append":
            return {"q": q, **pool}
    S, Pos, tab = pool["scores"].cpu().numpy(), pool["positions"].cpu().numpy(), table.cpu().numpy()
    at = {"from": [], "to": []}
    for b, n in enumerate(lens):
        L, m = past[b] + n, min(past[b] + n, c["budget"])
        recent = past[b] + n - c["recent"]                             # start equals past here
        home = tab[b, np.arange(L) // ps]
        into = s["dst_table"].cpu().numpy()[b] if c["fresh"] else tab[b]
        for h in range(c["H"]):
            sc, pos = S[home, h, np.arange(L) % ps], Pos[home, h, np.arange(L) % ps]
            worst_first = np.lexsort((pos, sc, pos >= recent))
            stay = np.sort(worst_first[L - m:])
            if c["fresh"]:
                frm, to = stay, np.arange(m)
            else:
                frm, to = stay[stay >= m], np.setdiff1d(np.arange(m), stay)
            at["from"].append(np.stack([home[frm], np.full(len(frm), h), frm % ps], 1))
            at["to"].append(np.stack([into[to // ps], np.full(len(to), h), to % ps], 1))
    frm, to = (torch.from_numpy(np.concatenate(at[x])).long().cuda().unbind(1) for x in ("from", "to"))
    for x in pool:
        pool[x][to] = pool[x][frm].clone()
    both = torch.tensor([[min(past[b] + n, c["budget"]), past[b] + n] for b, n in enumerate(lens)], dtype=torch.int32)
    return {**pool, "past_out": both[:, 0], "start_out": both[:, 1]}
