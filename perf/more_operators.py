"""Cases, plain forms and 64-bit definitions of rotary positions with several axes and of windowed attention over the paged cache.

Four operators that a serving program with images or video, or with layers of bounded reach, uses in this order, on [B][H][n][d] tensors:

  axes     y = m * (x rotated): pair k of a row turns by  position[axis of k] * f_k ; the axes are, say, time, height and width.
           (the transposed rotation is its gradient)
  append   rotates a chunk's queries and keys so and writes keys and values into the pages of a cache
  window   attention of the chunk over its cache pages: the row at slot p sees slots 0 .. sinks-1 and p-window+1 .. p ; and log-sum-exp
  slide    ends a step of such a cache: past and start move on, and pages that no later row sees leave the page table

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
        # queries of prompts full of images before a dense prefill, time / height / width: the largest tensor of the workloads
        dict(name="axes_prompt", op="axes", B=32, H=40, n=4096, d=128, dtype="bf16", pairs="16,24,24", cycle=False, each=False,
             interleaved=False, scaling="none", start=0, ragged=False, transpose=False),
        # gradient of partly rotated heads, two axes dealt in turn with frequencies of their own, neighbouring pairs, odd length, 32-bit storage
        dict(name="axes_grad", op="axes", B=4, H=12, n=1023, d=64, dtype="fp32", pairs="9,7", cycle=True, each=True,
             interleaved=True, scaling="linear", start=70001, ragged=True, transpose=True),
        # one token of every sequence enters the cache behind its images: latency
        dict(name="append_token_axes", op="append", B=32, H=40, G=1, d=128, dtype="bf16", ps=64, past=511, c=1, ragged=True,
             pairs="24,20,20", cycle=True, each=False, interleaved=False, scaling="none", start=511),
        # a ragged batch of prompt chunks with images behind a cached prefix, grouped heads
        dict(name="append_chunk_axes", op="append", B=8, H=8, G=4, d=128, dtype="fp16", ps=32, past=1000, c=2047, ragged=True,
             pairs="16,24,24", cycle=False, each=False, interleaved=False, scaling="bands", start=1000),
        # one token over a short window behind a long conversation whose old pages are gone: the smallest call
        dict(name="window_token_small", op="window", B=1, H=32, G=1, d=128, dtype="bf16", ps=16, past=5000, c=1, ragged=False,
             window=205, sinks=4, released=True),
        # one token of every sequence, ragged lengths around the window: bound by the bytes of what is seen
        dict(name="window_token_full", op="window", B=32, H=40, G=1, d=128, dtype="bf16", ps=64, past=8190, c=1, ragged=True,
             window=2048, sinks=4, released=False),
        # four drafted tokens behind long prompts, grouped heads
        dict(name="window_draft_long", op="window", B=8, H=8, G=4, d=128, dtype="fp16", ps=64, past=32700, c=4, ragged=False,
             window=4096, sinks=128, released=True),
        # a chunk of a long prompt: bound by the matrix products
        dict(name="window_chunk_long", op="window", B=1, H=32, G=1, d=128, dtype="bf16", ps=128, past=30720, c=2048, ragged=False,
             window=4096, sinks=4, released=True),
        # whole prompts in one chunk, grouped heads, a window of a quarter of the longest
        dict(name="window_prompt_group", op="window", B=8, H=8, G=4, d=128, dtype="fp16", ps=64, past=0, c=2048, ragged=True,
             window=512, sinks=16, released=False),
        # a small 32-bit prompt of odd length, heads of 64, an odd window that ends inside pages
        dict(name="window_prompt_fp32", op="window", B=2, H=4, G=1, d=64, dtype="fp32", ps=16, past=0, c=129, ragged=False,
             window=50, sinks=3, released=False),
        # the end of a generation step of a batch: a page or none leaves each table
        dict(name="slide_step", op="slide", B=32, ps=64, past=8190, c=1, ragged=True, window=2048, sinks=4),
        # the end of a long prompt of many sequences in small pages: thousands of pages leave
        dict(name="slide_prompt", op="slide", B=256, ps=16, past=0, c=32768, ragged=True, window=1024, sinks=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["axes", "append", "window", "window", "window", "slide"])
    ps, ragged = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    window, sinks = _log(rng, 1, 8192), rng.choice([0, 1, 4, 17, 64, 130])
    if op == "slide":
        return dict(op=op, B=_log(rng, 1, 256), ps=ps, past=rng.choice([0, _log(rng, 1, 32768)]), c=_log(rng, 1, 32768), ragged=ragged, window=window, sinks=sinks)
    dtype, d = rng.choice(["fp32", "bf16", "bf16", "fp16"]), rng.choice([64, 128])
    most, A, each = rng.choice([d // 2, d // 2, d // 4, 12, 8]), rng.choice([2, 3, 3, 4]), rng.random() < 0.4
    cuts = sorted(rng.sample(range(1, most), A - 1))
    pairs = ",".join(str(y - x) for x, y in zip([0] + cuts, cuts + [most]))
    angles = dict(pairs=pairs, cycle=rng.random() < 0.5, each=each, interleaved=rng.random() < 0.5,
                  scaling=rng.choice(["none", "linear"] if each else ["none", "linear", "ntk", "bands", "ramp"]), start=_log(rng, 1, 1000000))
    if op == "axes":
        B, H, n = _log(rng, 1, 32), _log(rng, 1, 40), _log(rng, 1, 4096)
        return dict(op=op, B=B, H=H, n=n, d=d, dtype=dtype, **angles, ragged=ragged, transpose=rng.random() < 0.5)
    H, G = _log(rng, 1, 32), rng.choice([1, 1, 2, 4, 5, 8])
    if op == "append":
        B, c = _log(rng, 1, 32), _log(rng, 1, 2048)
        B, H = (min(B, 8), min(H, 8)) if c > 256 else (B, H)
        return dict(op=op, B=B, H=H, G=G, d=d, dtype=dtype, ps=ps, past=_log(rng, 1, 2000), c=c, ragged=ragged, **angles)
    c, past = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 2048)]), rng.choice([0, _log(rng, 1, 32768), _log(rng, 1, 32768)])
    B = _log(rng, 1, 32)
    dense = 2 ** 24 if dtype == "fp32" else 2 ** 29               # logits of the call: fp32 storage is for small models
    rows = 2 ** 21 if dtype == "fp32" else 2 ** 22                # cached rows of the call
    while B * H * G * c * min(past + c, window + sinks + c) > dense or B * H * (past + c) > rows:
        if max(B, H) > 1:
            B, H = (B // 2, H) if B >= H else (B, H // 2)
        elif c > 1:
            c = c // 2
        else:
            past = past // 2
    return dict(op=op, B=B, H=H, G=G, d=d, dtype=dtype, ps=ps, past=past, c=c, ragged=ragged, window=window, sinks=sinks, released=rng.random() < 0.5)


# ---- what the cases say, as numbers -------------------------------------------------------------------------------

def _spread(most, B, ragged, shift):
    """Lengths of the batch: all `most`, or spread over 0 .. most (the first one is the longest)."""
    return [int(most * (1.0 - 0.95 * ((b * 0.6180339887 + shift * b) % 1.0))) if ragged else most for b in range(B)]


def _lens(c):
    n = c["n"] if c["op"] == "axes" else c["c"]
    return _spread(n, c["B"], c["ragged"] and n > 1, 0.37)


def _past(c):
    return _spread(c["past"], c["B"], c["ragged"], 0.0)


def _pairs(c):
    return [int(x) for x in c["pairs"].split(",")]


def _angles(c):
    """Axis of each pair, its frequency (64 bits), magnitude, and what the plans are made of."""
    pairs, scaling, theta0 = _pairs(c), c["scaling"], 10000.0
    deal = [(j, a) for a, n in enumerate(pairs) for j in range(n)]         # (index in its axis, axis), axis by axis
    deal = sorted(deal) if c["cycle"] else deal                            # or dealt in turn, axes that are full passed over
    axis = np.array([a for _, a in deal])
    r, factor, L = 2 * len(deal), 1.0 if scaling == "none" else 8.0, 4096
    made = dict(theta=theta0, interleaved=c["interleaved"], scaling=scaling, factor=factor, original_length=L, low=1.0, high=32.0 if scaling == "ramp" else 4.0)
    if c["each"]:                                                          # every axis has the whole range of frequencies
        f = np.array([theta0 ** (-j / pairs[a]) for j, a in deal]) / factor
        return axis, f, 1.0, [dict(made, rotary_dim=2 * n) for n in pairs]
    i = np.arange(r // 2, dtype=np.float64)
    theta = theta0 * factor ** (r / (r - 2.0)) if scaling == "ntk" else theta0
    f = theta ** (-2.0 * i / r)
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":
        t = np.clip((L * f / (2.0 * math.pi) - made["low"]) / (made["high"] - made["low"]), 0.0, 1.0)
        f = (1.0 - t) * f / factor + t * f
    if scaling == "ramp":
        at = [r * math.log(L / (2.0 * math.pi * beta)) / (2.0 * math.log(theta)) for beta in (made["high"], made["low"])]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        t = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        f = t * f / factor + (1.0 - t) * f
    return axis, f, (0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0), [dict(made, rotary_dim=r)]


def _first(past, window):
    """First slot within the window of the chunk's first row."""
    return max(0, past + 1 - window)


def work(c):
    if c["op"] == "slide":
        mp = -(-(c["past"] + c["c"]) // c["ps"])
        gone = sum(max(0, (p + n - c["window"] + 1) // c["ps"] - -(-c["sinks"] // c["ps"])) for p, n in zip(_past(c), _lens(c)))
        return {"bytes": c["B"] * (8 * mp + 24) + 4 * gone, "flops": 0}
    e, d = BYTES[c["dtype"]], c["d"]
    if c["op"] == "axes":
        rows = c["H"] * sum(_lens(c))
        return {"bytes": 2 * rows * d * e + 4 * len(_pairs(c)) * sum(_lens(c)), "flops": 6 * rows * sum(_pairs(c))}
    H, G, lens, past = c["H"], c["G"], _lens(c), _past(c)
    if c["op"] == "append":
        rows = H * sum(lens)
        return {"bytes": rows * ((4 + 2 * G) * d * e + 8) + 4 * len(_pairs(c)) * sum(lens), "flops": 6 * rows * (G + 1) * sum(_pairs(c))}
    W, S = c["window"], c["sinks"]
    seen = pairs = 0
    for p, n in zip(past, lens):
        if n:
            lo = _first(p, W)
            seen += p + n - lo + min(S, lo)
            i = np.arange(n, dtype=np.int64) + p
            pairs += int((np.minimum(i + 1, W) + np.minimum(S, np.maximum(i + 1 - W, 0))).sum())
    rows = sum(H * G * n for n in lens)
    return {"bytes": H * seen * 2 * d * e + rows * (2 * d * e + 4), "flops": 4 * d * H * G * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _normal(gen, shape, dtype):
    return torch.randn(shape, dtype=dtype if dtype != torch.float32 else None, device="cuda", generator=gen)


def _places(c, gen, n):
    """Positions [axes][B][n] of prompts that are text and images in turn: a text token stands at the same place on every axis, an image's
    patches at one time and at their row and column (and, on a fourth axis, at the image's number)."""
    A, B = len(_pairs(c)), c["B"]
    shift = torch.randint(0, 50, (B, 1), generator=gen, device="cuda")
    t = torch.arange(n, device="cuda").expand(B, n) + shift
    block, at = t // 240, t % 240                                 # 40 tokens of text, then 200 patches of 10 x 20
    base = block * 60 + c["start"] + 17 * torch.arange(B, device="cuda")[:, None]
    image, patch = at >= 40, at - 40
    axes = [base + 40, base + 40 + patch // 20, base + 40 + patch % 20, block]
    rows = [torch.where(image, x, base + at) for x in axes]
    return torch.stack(rows[:A] if A > 2 else rows[1:3]).to(torch.int32).contiguous()      # two axes: height and width


def _cache(c, gen, slots):
    """Pool, page table (pages in no order) and lengths; every slot of the pool holds something."""
    B, H, d, ps, dt = c["B"], c["H"], c["d"], c["ps"], DTYPES[c["dtype"]]
    mp = -(-slots // ps)
    past = _past(c)
    keep = torch.ones((B, mp), dtype=torch.bool, device="cuda")
    if c.get("released"):                                          # pages that no row of the call sees have left the table
        page = torch.arange(mp, device="cuda")
        lo = _int([_first(p, c["window"]) for p in past])[:, None]
        keep = (page * ps < c["sinks"]) | ((page + 1) * ps > lo)
    pages = int(keep.sum()) + 1
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, mp), -1, dtype=torch.int32, device="cuda")
    table[keep] = order[: pages - 1]
    s = dict(k_pages=_normal(gen, (pages, H, ps, d), dt), v_pages=_normal(gen, (pages, H, ps, d), dt), page_table=table,
             past=_int(past), start=_int(past), lens=_int(_lens(c)))
    s["k_pages"][table[:, 0].clamp_min(0).long(), :, 0] *= 4          # the first token of a sequence draws attention
    s["scores"] = torch.rand((pages, H, ps), device="cuda", generator=gen)
    s["positions"] = torch.full((pages, H, ps), -1, dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if c["op"] == "slide":
        B, mp = c["B"], -(-(c["past"] + c["c"]) // c["ps"])
        s = dict(case=c, page_table=torch.randperm(B * mp, generator=gen, device="cuda").to(torch.int32).view(B, mp), past=_int(_past(c)), lens=_int(_lens(c)))
        s["start"] = s["past"] + 9
        s["out"] = {"table": torch.zeros_like(s["page_table"]), "freed": torch.full_like(s["page_table"], -5),
                    **{x: torch.zeros_like(s["past"]) for x in ("freed_count", "past", "start")}}
        if own:                                                    # a table's pages are what counts: one head of few elements stands for the layers
            from paper_2407_20485_b200 import binding as a2sf
            s["cache"] = a2sf.PagedCache(B, 1, 64, torch.bfloat16, c["ps"], B * mp, mp, page_table=s["page_table"], past=s["past"], start=s["start"])
        return s
    dt, d = DTYPES[c["dtype"]], c["d"]
    if c["op"] == "axes":
        x = _normal(gen, (c["B"], c["H"], c["n"], d), dt)
        s = dict(x=x, out=torch.zeros_like(x), lens=_int(_lens(c)), places=_places(c, gen, c["n"]))
    else:
        B, H, G, n = c["B"], c["H"], c["G"], c["c"]
        s = _cache(c, gen, c["past"] + n)
        s["q"] = _normal(gen, (B, H * G, n, d), dt)
        s["out"] = torch.zeros_like(s["q"])
        if c["op"] == "append":
            s["k"], s["v"] = _normal(gen, (B, H, n, d), dt), _normal(gen, (B, H, n, d), dt)
            s["start"] = s["start"] + 7
            s["places"] = _places(c, gen, n)
        else:
            s["lse"] = torch.zeros((B, H * G, n), dtype=torch.float32, device="cuda")
    s["case"] = c
    if "pairs" in c:
        axis, f, s["magnitude"], plans = _angles(c)
        s["axis"], s["inv_freq"] = torch.from_numpy(axis).cuda(), torch.from_numpy(f).cuda()
    if own:                                                        # the handles that a program keeps
        from paper_2407_20485_b200 import binding as a2sf
        if "pairs" in c:
            s["plan"] = a2sf.a2sf_rotary_axes_plan_init(_pairs(c), [a2sf.a2sf_rotary_plan_init(**p) for p in plans], cycle=c["cycle"])
        if c["op"] != "axes":
            s["cache"] = a2sf.PagedCache(c["B"], c["H"], d, dt, c["ps"], s["k_pages"].shape[0], s["page_table"].shape[1], group=c["G"],
                                         **{k: s[k] for k in ("k_pages", "v_pages", "scores", "positions", "page_table", "past", "start")})
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _rotated(s, x, transpose=False):
    """x [B][H][n][d] rotated: angles in 64 bits, arithmetic in 32, one rounding."""
    half = s["inv_freq"].numel()
    ang = s["places"][s["axis"]].permute(1, 2, 0)[:, None].double() * s["inv_freq"]        # [B][1][n][pairs]
    cos, sin = (torch.cos(ang) * s["magnitude"]).float(), (torch.sin(ang) * s["magnitude"]).float()
    if transpose:
        sin = -sin
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["case"]["interleaved"] else (slice(0, half), slice(half, 2 * half))
    x1, x2 = x[..., a].float(), x[..., b].float()
    y = x.clone()
    y[..., a] = (x1 * cos - x2 * sin).to(x.dtype)
    y[..., b] = (x2 * cos + x1 * sin).to(x.dtype)
    return y


def _live(s):
    n = s["out"].shape[2]
    return torch.arange(n, device="cuda") < s["lens"][:, None]                              # [B][n]


def _axes(s):
    return {"out": torch.where(_live(s)[:, None, :, None], _rotated(s, s["x"], s["case"]["transpose"]), s["out"])}


def _append(s):
    """Writes rotated keys, and values, where they belong; scores start at zero."""
    ps, live = s["case"]["ps"], _live(s)
    k, q = _rotated(s, s["k"]), _rotated(s, s["q"])
    b, i = torch.nonzero(live, as_tuple=True)
    slot = s["past"].long()[b] + i
    page, off = s["page_table"].long()[b, slot // ps], slot % ps
    s["k_pages"][page, :, off] = k[b, :, i]
    s["v_pages"][page, :, off] = s["v"][b, :, i]
    s["scores"][page, :, off] = 0.0
    s["positions"][page, :, off] = (s["start"][b] + i.to(torch.int32))[:, None].expand(-1, k.shape[1])
    return {"q": torch.where(live[:, None, :, None], q, s["out"]), **{x: s[x] for x in ("k_pages", "v_pages", "scores", "positions")}}


def _window(s):
    """Only what some row of the call may see is gathered: the sinks, and the windows of all rows as one range."""
    c = s["case"]
    B, H, G, d, n, ps, W, S = c["B"], c["H"], c["G"], c["d"], c["c"], c["ps"], c["window"], c["sinks"]
    past, live, i = s["past"].long()[:, None], _live(s), torch.arange(n, device="cuda")
    lo = (past + 1 - W).clamp_min(0)                                                       # [B][1]
    most = s["page_table"].shape[1] * ps
    early = torch.arange(min(S, most), device="cuda").expand(B, -1)
    late = lo + torch.arange(min(W - 1 + n, most), device="cuda")
    j = torch.cat([torch.where(early < lo, early, most), late], 1)                          # slots; `most` is none
    page = torch.gather(s["page_table"].long(), 1, (j // ps).clamp_max(most // ps - 1)).clamp_min(0)
    kv = [x[page, :, j % ps].transpose(1, 2).float() for x in (s["k_pages"], s["v_pages"])]  # [B][H][slots][d]
    at = (past + i)[:, :, None]
    seen = (j[:, None] <= at) & ((j[:, None] > at - W) | (j[:, None] < S)) & (j[:, None] < most) & live[:, :, None]      # [B][n][slots]
    x = torch.matmul(s["q"].float().view(B, H, G * n, d), kv[0].transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, H, G, n, -1)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min_(-3.0e38)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    x = x.div_(total.clamp_min(1e-38))
    out = torch.matmul(x.view(B, H, G * n, -1), kv[1]).view(B, H * G, n, d).to(s["out"].dtype)
    lse = (m + torch.log(total)).view(B, H * G, n)
    mask = live[:, None, :]
    return {"out": torch.where(mask[..., None], out, s["out"]), "lse": torch.where(mask, lse, s["lse"])}


def _slide(s):
    c, o, table = s["case"], s["out"], s["page_table"]
    n = s["past"] + s["lens"]
    page = torch.arange(table.shape[1], device="cuda")
    gone = (page * c["ps"] >= c["sinks"]) & ((page + 1) * c["ps"] <= (n - c["window"] + 1)[:, None]) & (table >= 0)
    o["table"].copy_(torch.where(gone, -1, table))
    at = torch.cumsum(gone, 1) - 1
    b, p = torch.nonzero(gone, as_tuple=True)
    o["freed"][b, at[b, p]] = table[b, p]
    o["freed_count"].copy_(gone.sum(1))
    o["past"].copy_(n)
    o["start"].copy_(s["start"] + s["lens"])
    return o


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"axes": _axes, "append": _append, "window": _window, "slide": _slide}[c["op"]](s)
    if c["op"] == "axes":
        from paper_2407_20485_b200 import binding as a2sf
        return {"out": a2sf.a2sf_rotary_axes(s["plan"], s["x"], s["places"], out=s["out"], lens=s["lens"], transpose=c["transpose"])}
    cache = s["cache"]
    if c["op"] == "append":
        q = cache.a2sf_paged_append_axes(s["k"], s["v"], s["places"], s["plan"], lens=s["lens"], q=s["q"], q_out=s["out"])
        return {"q": q, **{x: s[x] for x in ("k_pages", "v_pages", "scores", "positions")}}
    if c["op"] == "window":
        out, lse = cache.a2sf_paged_attend_window(s["q"], c["window"], c["sinks"], lens=s["lens"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    o = s["out"]
    cache.a2sf_paged_slide(c["window"], c["sinks"], c["c"], lens=s["lens"], table_out=o["table"], freed=o["freed"], freed_count=o["freed_count"],
                           past_out=o["past"], start_out=o["start"])
    return o


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def _turn(x, places, c):
    """x [H][n][d] in 64 bits at places [axes][n], pair by pair as complex numbers."""
    axis, f, m, _ = _angles(c)
    h = len(f)
    z = torch.stack([places[a].double() * w for a, w in zip(axis.tolist(), f.tolist())], 1)
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
    if c["op"] == "axes":
        out = s["out"].double()
        for b, n in enumerate(lens):
            out[b, :, :n] = _turn(s["x"][b, :, :n].double(), s["places"][:, b, :n], c)
        return {"out": out}
    past, ps, tab = _past(c), c["ps"], s["page_table"].cpu().numpy()
    if c["op"] == "slide":
        o = {x: y.cpu().numpy() for x, y in s["out"].items()}
        o["table"] = tab.copy()
        for b, n in enumerate(lens):
            end = past[b] + n
            leave = [p for p in range(-(-c["sinks"] // ps), tab.shape[1]) if p * ps + ps - 1 <= end - c["window"]]
            o["freed"][b, : len(leave)] = tab[b, leave]
            o["table"][b, leave] = -1
            o["freed_count"][b], o["past"][b], o["start"][b] = len(leave), end, past[b] + 9 + n
        return o
    table = s["page_table"].long()
    if c["op"] == "append":
        pool = {x: s[x].double() if s[x].is_floating_point() else s[x] for x in ("k_pages", "v_pages", "scores", "positions")}
        q = s["out"].double()
        for b, n in enumerate(lens):
            if not n:
                continue
            at = torch.arange(n, device="cuda")
            pg, off = table[b, (past[b] + at) // ps], (past[b] + at) % ps
            q[b, :, :n] = _turn(s["q"][b, :, :n].double(), s["places"][:, b, :n], c)
            pool["k_pages"][pg, :, off] = _turn(s["k"][b, :, :n].double(), s["places"][:, b, :n], c).transpose(0, 1)
            pool["v_pages"][pg, :, off] = s["v"][b, :, :n].double().transpose(0, 1)
            pool["scores"][pg, :, off] = 0.0
            pool["positions"][pg, :, off] = (at + past[b] + 7).to(torch.int32)[:, None]
        return {"q": q, **pool}
    G, H, W, S = c["G"], c["H"], c["window"], c["sinks"]
    out, lse = s["out"].double(), s["lse"].double()
    for b, n in enumerate(lens):
        for i0 in range(0, n, 256):                                  # rows of a block and all that they see
            i1 = min(n, i0 + 256)
            lo, end = max(0, past[b] + i0 - W + 1), past[b] + i1
            slot = torch.cat([torch.arange(min(S, lo), device="cuda"), torch.arange(lo, end, device="cuda")])
            K, V = (s[x][table[b, slot // ps], :, slot % ps].double().transpose(0, 1) for x in ("k_pages", "v_pages"))
            row = torch.arange(past[b] + i0, end, device="cuda")[:, None]
            hidden = (slot > row) | ((slot >= S) & (slot + W <= row))
            x = torch.einsum("hgnd,hjd->hgnj", s["q"][b, :, i0:i1].double().reshape(H, G, i1 - i0, -1), K) / math.sqrt(c["d"])
            x.masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(x, 3)
            out[b, :, i0:i1] = torch.einsum("hgnj,hjd->hgnd", torch.exp(x - z[..., None]), V).reshape(H * G, i1 - i0, -1)
            lse[b, :, i0:i1] = z.reshape(H * G, -1)
    return {"out": out, "lse": lse}
