"""Windowed attention over the paged cache, and the pages that leave it, against plain 64-bit forms on a B200.

Tolerances count roundings as in the tests of the attention without a window: u is the half step of the storage type, f = 2^-24.
A logit is off by at most e = (d + 2) f sum|q k| scale, a probability by 2 e + 2^-20 of itself; the row sums over the slots seen."""
import math
import random

import pytest
import torch

import paged_util as pu

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import binding

    return binding


@pytest.fixture(autouse=True)
def _clean_status(a2sf):
    a2sf.a2sf_last_device_status()
    yield
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK


def close(got, want, tol, what):
    got, want = got.double().cpu(), want.double()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float(((got - want).abs() / tol.clamp_min(1e-300)).nan_to_num(math.inf).max()):.3g} of the tolerance")


def window_ref(K, V, q, past, window, sinks, scale):
    """One sequence and K/V head in 64 bits: K, V [L][d], q [G][n][d] -> out, lse, sum P|V|, logit size, slots of the longest row."""
    n, L = q.shape[1], K.shape[0]
    p, j = past + torch.arange(n)[:, None], torch.arange(L)[None, :]
    seen = (j <= p) & ((j < sinks) | (j > p - window))
    use = seen.any(0)                                          # slots that no row sees may hold anything
    K, V = torch.where(use[:, None], K, 0.0), torch.where(use[:, None], V, 0.0)
    x = torch.einsum("gnd,ld->gnl", q, K) * scale
    size = float((torch.einsum("gnd,ld->gnl", q.abs(), K.abs()) * scale).masked_fill(~seen, 0.0).max())
    x = x.masked_fill(~seen, -math.inf)
    z = torch.logsumexp(x, -1)
    P = torch.exp(x - z[..., None])
    return P @ V, z, P @ V.abs(), size, int(seen.sum(1).max()), float(V.abs().max())


def hide(cache, past, window, sinks, bad, table=True):
    """What no row of a chunk behind ``past`` sees holds ``bad``; pages of it alone leave the table."""
    ps = cache.page_size
    t = cache.page_table.cpu()
    k, v = cache.k_pages.cpu(), cache.v_pages.cpu()
    for b, p in enumerate(past):
        lo = max(0, p + 1 - window)
        for j in range(min(sinks, lo), lo):
            k[int(t[b, j // ps]), :, j % ps] = bad
            v[int(t[b, j // ps]), :, j % ps] = bad
        for e in range(t.shape[1]) if table else ():
            if e * ps >= sinks and (e + 1) * ps <= lo:
                t[b, e] = -1
    cache.k_pages.copy_(k), cache.v_pages.copy_(v), cache.page_table.copy_(t)


def check_window(a2sf, case, seed=5, garbage=float("nan"), gain=1.0, room=0):
    B, H, G, d, dtype, ps, past, c, lens, window, sinks, layout, scale = case
    lens = [c] * B if lens is None else lens
    cache = pu.make_cache(a2sf, B, H, G, d, dtype, ps, past, max(c, room), seed=seed, scale=scale, garbage=garbage)
    g = torch.Generator().manual_seed(seed + 1)

    def tensor(h, k=1.0):
        t = (torch.randn((B, h, c, d), generator=g) * k).to(dtype)
        return t, (t.cuda() if layout == "bhnd" else t.transpose(1, 2).contiguous().cuda().transpose(1, 2))

    (k, kc), (v, vc), (q, qc) = tensor(H), tensor(H), tensor(H * G, gain)
    L = torch.tensor(lens, dtype=I32).cuda()
    whole = cache.page_table.cpu().clone()
    cache.a2sf_paged_append(kc, vc, lens=L)
    hide(cache, past, window, sinks, garbage)
    pool = {x: getattr(cache, x).cpu().clone() for x in ("k_pages", "v_pages", "scores", "positions")}
    out, lse = torch.full_like(qc, 3.0), torch.full((B, H * G, c), 3.0, device="cuda")
    # the binding's torch: in the debug sweep it puts guard words around the workspace
    cache.a2sf_paged_attend_window(qc, window, sinks, lens=L, out=out, lse=lse, workspace=a2sf.torch.empty(
        (cache.attend_window_workspace_bytes(c, window, sinks),), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for x, t in pool.items():
        assert torch.equal(getattr(cache, x).cpu().double().nan_to_num(7.0, 8.0), t.double().nan_to_num(7.0, 8.0)), f"{x} changed"
    sc, u = scale or 1 / math.sqrt(d), torch.finfo(dtype).eps / 2
    view = cache.page_table.cpu().clone()
    cache.page_table.copy_(whole)                              # for the reference, which masks
    K, V = pool["k_pages"].double(), pool["v_pages"].double()
    for b in range(B):
        n = lens[b]
        assert bool((out[b, :, n:] == 3.0).all()) and bool((lse[b, :, n:] == 3.0).all()), "rows past the length were written"
        if n == 0:
            continue
        Kb, Vb = (pu.slots(cache, x, b, past[b] + n) for x in (K, V))
        for h in range(H):
            o, z, size, logit, most, vmax = window_ref(Kb[h], Vb[h], q[b, h * G:(h + 1) * G, :n].double(), past[b], window, sinks, sc)
            e = (d + 2) * F * logit
            rel = 2 * e + 2.0 ** -20
            # fp16: 2^-25 absolutely below its normal range, against a row sum of at least 1
            under = 0.0 if dtype != HF else 2.0 ** -25 * most * vmax
            close(out[b, h * G:(h + 1) * G, :n], o, u * o.abs() + (u + rel + most * F) * size + under, f"out {b} {h}")
            close(lse[b, h * G:(h + 1) * G, :n], z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), f"lse {b} {h}")
    cache.page_table.copy_(view)
    return cache, qc, L, out, lse


WIN = [
    # B, H, G, d, dtype, ps, past, c, lens, window, sinks, layout, scale
    (1, 1, 1, 64, FP, 16, [0], 1, None, 1, 0, "bhnd", 0.0),                     # one token, nothing before it, itself alone
    (1, 1, 1, 64, BF, 16, [40], 1, None, 1, 0, "bhnd", 0.0),                    # itself alone behind 40
    (2, 2, 1, 64, FP, 16, [0, 0], 129, None, 50, 3, "bhnd", 0.0),
    (3, 2, 3, 128, FP, 32, [70, 0, 5], 33, [33, 0, 20], 17, 40, "bnhd", 0.2),   # more sinks than some sequences have slots
    (2, 1, 8, 128, FP, 64, [1000, 33], 1, [1, 0], 300, 0, "bhnd", 0.0),
    (2, 3, 5, 64, FP, 128, [200, 64], 70, [70, 69], 1, 1, "bnhd", 0.0),
    (4, 3, 1, 128, BF, 16, [204, 0, 63, 64], 1, None, 64, 4, "bhnd", 0.0),      # few rows
    (5, 2, 1, 128, BF, 64, [130, 7, 500, 0, 1], 1, [1, 0, 1, 1, 1], 100, 17, "bhnd", 0.0),
    (2, 2, 4, 128, HF, 64, [1999, 17], 4, [4, 3], 700, 5, "bnhd", 0.0),
    (2, 2, 8, 64, HF, 32, [333, 100], 1, None, 33, 64, "bhnd", 0.0),
    (1, 3, 8, 128, BF, 128, [640], 2, None, 2, 130, "bhnd", 0.3),
    (3, 1, 5, 64, BF, 16, [37, 0, 90], 3, [3, 2, 0], 2, 0, "bnhd", 0.0),         # rows of a call with windows apart
    (1, 2, 3, 128, HF, 16, [9000], 5, None, 4000, 31, "bhnd", 0.0),             # one long sequence
    (2, 1, 2, 64, BF, 64, [4096, 4095], 1, None, 4096, 0, "bhnd", 0.0),         # exactly the window, and one slot short of it
    (2, 1, 16 // 4, 128, BF, 16, [500, 20], 4, None, 100000, 100000, "bhnd", 0.0),       # nothing is left out
    (1, 1, 1, 128, HF, 16, [0], 17, None, 5, 0, "bhnd", 0.0),                   # many rows
    (2, 2, 1, 128, BF, 64, [0, 0], 128, [128, 127], 30, 4, "bhnd", 0.0),
    (2, 2, 4, 128, HF, 32, [0, 300], 200, [200, 77], 64, 16, "bnhd", 0.0),
    (3, 1, 5, 128, BF, 16, [511, 0, 129], 100, [100, 0, 51], 200, 0, "bhnd", 0.0),
    (1, 2, 8, 64, HF, 128, [1000], 129, None, 1, 3, "bhnd", 0.0),
    (2, 1, 3, 64, BF, 64, [0, 77], 300, [300, 1], 100, 129, "bnhd", 0.25),
    (1, 1, 7, 128, BF, 16, [2500], 41, None, 1000, 7, "bhnd", 0.0),
    (2, 3, 1, 128, HF, 128, [640, 1], 513, [513, 512], 128, 0, "bhnd", 0.0),
]
MANY = [                                                                       # few rows of more units than fit at once, and long windows of few units
    (40, 8, 1, 128, BF, 16, [300 + 7 * (b % 9) for b in range(40)], 1, [b % 5 and 1 for b in range(40)], 100, 5, "bhnd", 0.0),
    (40, 8, 2, 64, HF, 64, [90 + 100 * (b % 8) for b in range(40)], 3, [3, 2, 0, 1] * 10, 700, 33, "bnhd", 0.0),
    (20, 8, 1, 128, FP, 32, [600 - 29 * b for b in range(20)], 1, None, 250, 20, "bhnd", 0.0),
    (20, 9, 4, 64, FP, 16, [b * 20 for b in range(20)], 2, [2, 1, 0, 2, 2] * 4, 90, 0, "bnhd", 0.0),
    (100, 3, 4, 128, BF, 16, [20 * (b % 30) for b in range(100)], 4, [4, 0, 3, 1] * 25, 64, 16, "bhnd", 0.0),
    (1, 2, 3, 128, HF, 16, [9000], 5, None, 7000, 31, "bhnd", 0.0),
    (1, 3, 2, 64, FP, 32, [5000], 4, None, 4000, 1, "bnhd", 0.0),
]
LARGE = [                                                                      # tcgen05: direct, and with pieces and merge
    (4, 12, 2, 128, BF, 16, [0, 700, 3, 1500], 400, [400, 399, 0, 130], 150, 4, "bnhd", 0.0),
    (4, 12, 2, 64, HF, 128, [0, 700, 3, 1500], 400, [400, 1, 77, 256], 1, 0, "bhnd", 0.0),
    (2, 16, 1, 128, HF, 64, [3000, 100], 300, [300, 300], 2000, 0, "bhnd", 0.0),
    (1, 8, 4, 128, BF, 32, [6000], 200, None, 5000, 100, "bhnd", 0.0),
    (1, 8, 1, 64, BF, 128, [9000], 1000, None, 3500, 1, "bhnd", 0.0),
    (1, 5, 3, 128, HF, 16, [2000], 700, None, 129, 33, "bnhd", 0.0),
    (2, 6, 8, 128, BF, 64, [0, 50], 500, [500, 450], 100000, 0, "bhnd", 0.0),
    (6, 20, 1, 128, BF, 64, [0, 10, 2000, 0, 5, 1], 600, [600, 0, 600, 33, 599, 256], 500, 16, "bhnd", 0.0),
    (1, 4, 4, 128, HF, 64, [5000], 64, None, 4096, 4, "bhnd", 0.0),             # items longer than a part
    (2, 3, 8, 64, BF, 16, [9000, 20], 40, [40, 33], 8000, 0, "bnhd", 0.0),
    (60, 8, 1, 128, BF, 32, [b % 7 * 50 for b in range(60)], 130, [130 - 2 * b for b in range(60)], 40, 2, "bhnd", 0.0),      # rounds of whole items
]


def ident(c):
    return "-".join(str(x).replace("torch.", "").replace(" ", "")[:40] for x in c)


@pytest.mark.parametrize("case", WIN + MANY + LARGE, ids=ident)
def test_window(a2sf, case):
    cache, qc, L, out, lse = check_window(a2sf, case)
    # the same call again, without lse given: the same bits
    again, z = cache.a2sf_paged_attend_window(qc, case[9], case[10], lens=L, out=torch.full_like(out, 3.0), lse=torch.full_like(lse, 3.0))
    assert torch.equal(again, out) and torch.equal(z, lse)


@pytest.mark.parametrize("seed", range(60))
def test_window_random_cases(a2sf, seed):
    check_window(a2sf, random_window(random.Random(seed)), seed=seed + 100)


def random_window(r):
    B, H, G = r.choice([1, 1, 2, 3, 6]), r.choice([1, 2, 3]), r.choice([1, 1, 2, 3, 4, 5, 6, 7, 8])
    c = r.choice([1, 1, 2, 16 // G, 16 // G + 1, int(2 ** r.uniform(1, 9)), 128 // G, 256 // G + 1])
    past = [int(2 ** r.uniform(0, 10)) - 1 if r.random() < 0.9 else 0 for _ in range(B)]
    lens = [r.choice([c, c, c, 0, r.randint(0, c)]) for _ in range(B)]
    return (B, H, G, r.choice([64, 128]), r.choice([FP, BF, BF, HF]), r.choice([16, 32, 64, 128]), past, max(1, c), lens,
            r.choice([1, 2, 15, 16, 17, int(2 ** r.uniform(0, 10)), int(2 ** r.uniform(0, 10))]), r.choice([0, 0, 1, 4, 16, 31, 130]),
            r.choice(["bhnd", "bnhd"]), r.choice([0.0, 0.0, 0.2]))


@pytest.mark.parametrize("seed", range(24))
def test_window_random_large_calls(a2sf, seed):
    r = random.Random(1000 + seed)
    B, G = r.choice([1, 2, 4]), r.choice([1, 2, 3, 4, 8])
    H, c = r.choice([6, 10, 16]), r.choice([150, 300, 500, 900]) // min(G, 3)
    past = [int(2 ** r.uniform(0, 12)) - 1 for _ in range(B)]
    lens = [r.choice([c, c, 0, r.randint(0, c)]) for _ in range(B)]
    check_window(a2sf, (B, H, G, r.choice([64, 128]), r.choice([BF, HF]), r.choice([16, 32, 64, 128]), past, c, lens, int(2 ** r.uniform(0, 12)),
                        r.choice([0, 1, 4, 17, 130]), r.choice(["bhnd", "bnhd"]), r.choice([0.0, 0.2])), seed=seed + 300)


@pytest.mark.parametrize("dtype,G,c,past,window,sinks,gain,garbage", [
    (BF, 2, 1, 600, 100, 4, 12.0, "nan"), (HF, 2, 1, 600, 100, 0, 12.0, "inf"), (FP, 2, 1, 100, 33, 1, 12.0, "-inf"), (FP, 1, 40, 30, 9, 2, 12.0, "inf"),
    (BF, 1, 300, 200, 70, 0, 12.0, "inf"), (HF, 4, 150, 200, 130, 5, 12.0, "-inf"), (HF, 4, 4, 300, 50, 40, 12.0, "nan")])
def test_large_logits_and_what_no_row_sees(a2sf, dtype, G, c, past, window, sinks, gain, garbage):
    """Logits of +-100: a row's first visible tile sets its reference, whatever came before; infinities and NaN between sinks and window."""
    for H in (1, 12):
        check_window(a2sf, (2, H, G, 128, dtype, 32, [past, 0], c, None, window, sinks, "bhnd", 0.0), seed=9, gain=gain, garbage=float(garbage))


@pytest.mark.parametrize("dtype,c", [(BF, 300), (HF, 300), (BF, 40), (FP, 100), (HF, 2)])
def test_rows_whose_logits_are_all_far_below_zero(a2sf, dtype, c):
    """All logits -200 (log2 units -288) in most slots, 0 in a few: a row whose first visible tile holds only low ones keeps them."""
    H, d, past, window = 10, 128, 500, 140
    cache = a2sf.PagedCache(1, H, d, dtype, 64, 16, 16, scale=1.0)
    cache.page_table.copy_(torch.arange(16).view(1, -1))
    n = past + c
    k, v = torch.zeros((1, H, n, d), dtype=dtype), torch.randn((1, H, n, d), generator=torch.Generator().manual_seed(3)).to(dtype)
    k[..., 0] = -200.0
    k[0, :, 40, 0] = 0.0                                       # seen by the first rows of some windows only
    k[0, :, 450, 0] = 0.0
    q = torch.zeros((1, H, c, d), dtype=dtype)
    q[..., 0] = 1
    cache.a2sf_paged_append(k.cuda(), v.cuda())
    cache.past.fill_(past)
    for sinks in (0, 3, 41):
        out, lse = cache.a2sf_paged_attend_window(q.cuda(), window, sinks)
        o, z, size, logit, most, vmax = window_ref(k[0, 0].double(), v[0, 0].double(), q[0, :1].double(), past, window, sinks, 1.0)
        u, e = torch.finfo(dtype).eps / 2, (d + 2) * F * 200
        under = 0.0 if dtype != HF else 2.0 ** -25 * most * vmax
        close(out[0, :1], o, u * o.abs() + (u + 2 * e + 2.0 ** -20 + most * F) * size + under, f"out {sinks}")
        close(lse[0, :1], z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), f"lse {sinks}")


@pytest.mark.parametrize("dtype,G,c", [(BF, 1, 1), (HF, 4, 3), (FP, 2, 1), (FP, 1, 50), (BF, 2, 30), (BF, 1, 700), (HF, 8, 200)])
def test_a_window_of_everything_is_the_attention_without_one(a2sf, dtype, G, c):
    """Up to the cut of the work into pieces, which depends on what is seen: the same sums in another order."""
    B, H, d = 2, 6, 128
    cache = pu.make_cache(a2sf, B, H, G, d, dtype, 32, [90, 300], c, seed=3)
    g = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn((B, h, c, d), generator=g).to(dtype).cuda() for h in (H * G, H, H))
    cache.a2sf_paged_append(k, v)
    out, lse = cache.a2sf_paged_attend(q, scores=False)
    for window, sinks in ((2 ** 31 - 1, 0), (300 + c, 0), (1, 2 ** 31 - 1)):
        o, z = cache.a2sf_paged_attend_window(q, window, sinks)
        assert float((o.float() - out.float()).abs().max()) <= 4 * torch.finfo(dtype).eps / 2 * 4.5 + 1e-5
        assert float((z - lse).abs().max()) <= 2e-5


@pytest.mark.parametrize("chunks", [[40, 1, 1, 29], [1, 64, 5, 140, 2], [260, 10, 1, 1, 3]])
@pytest.mark.parametrize("dtype,G,d", [(BF, 1, 128), (HF, 4, 64), (FP, 2, 64)])
def test_steps_with_axes_window_and_slide_in_recycled_pages(a2sf, chunks, dtype, G, d):
    """A prompt in chunks and tokens from one small pool: append with three axes, attend, slide; freed pages are given out again.  Every
    row equals attention over all tokens so far."""
    B, H, ps, window, sinks, n = 2, 3, 16, 50, 20, sum(chunks)
    pairs = [d // 4, d // 8, d // 8]
    base = a2sf.a2sf_rotary_plan_init(d)
    plan = a2sf.a2sf_rotary_axes_plan_init(pairs, base)
    g = torch.Generator().manual_seed(17)
    q, k, v = (torch.randn((B, h, n, d), generator=g).to(dtype).cuda() for h in (H * G, H, H))
    pos = torch.randint(0, 500, (3, B, n), generator=g).to(I32).cuda()
    mp = -(-n // ps)
    free = list(range(B * (max(chunks) + window + sinks + 3 * ps) // ps + 4))
    random.Random(3).shuffle(free)
    cache = a2sf.PagedCache(B, H, d, dtype, ps, len(free), mp, group=G)
    cache.k_pages.fill_(float("nan")), cache.v_pages.fill_(float("nan"))
    at, u = 0, torch.finfo(dtype).eps / 2
    keys, queries = (a2sf.a2sf_rotary_axes(plan, x, pos) for x in (k, q))      # rounded as in the pages
    for c in chunks:
        part = slice(at, at + c)
        table = cache.page_table.cpu()
        for b in range(B):
            for e in range(at // ps, -(-(at + c) // ps)):
                if table[b, e] < 0:
                    table[b, e] = free.pop()
        cache.page_table.copy_(table)
        qr = cache.a2sf_paged_append_axes(k[:, :, part], v[:, :, part], pos[:, :, part].contiguous(), plan, q=q[:, :, part])
        assert torch.equal(qr, queries[:, :, part])
        out, lse = cache.a2sf_paged_attend_window(qr, window, sinks)
        for b in range(B):
            for h in range(H):
                o, z, size, logit, most, vmax = window_ref(keys[b, h, : at + c].double().cpu(), v[b, h, : at + c].double().cpu(),
                                                           qr[b, h * G:(h + 1) * G].double().cpu(), at, window, sinks, 1 / math.sqrt(d))
                e = (d + 2) * F * logit
                under = 0.0 if dtype != HF else 2.0 ** -25 * most * vmax
                close(out[b, h * G:(h + 1) * G], o, u * o.abs() + (u + 2 * e + 2.0 ** -20 + most * F) * size + under, f"out {at} {b} {h}")
                close(lse[b, h * G:(h + 1) * G], z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), f"lse {at} {b} {h}")
        freed, count = torch.full((B, mp), -9, dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
        cache.a2sf_paged_slide(window, sinks, c, freed=freed, freed_count=count)
        at += c
        for b in range(B):
            got = freed[b, : int(count[b])].tolist()
            free += got
            for pg in got:                                        # whoever gets them next writes what it needs
                cache.k_pages[pg].fill_(float("nan")), cache.v_pages[pg].fill_(float("nan"))
    assert cache.past.tolist() == [n] * B and cache.start.tolist() == [n] * B
    held = int((cache.page_table >= 0).sum())
    assert held + len(free) == cache.num_pages and len(set(free)) == len(free)
    assert held <= B * (-(-sinks // ps) + (window - 1) // ps + 2)


# ---- slide -----------------------------------------------------------------------------------------------

def slide_ref(table, n, ps, window, sinks):
    out, freed = table.clone(), []
    for b in range(table.shape[0]):
        gone = [e for e in range(table.shape[1]) if e * ps >= sinks and (e + 1) * ps <= n[b] - window + 1 and table[b, e] >= 0]
        freed.append([int(table[b, e]) for e in gone])
        out[b, gone] = -1
    return out, freed


@pytest.mark.parametrize("B,ps,mp,past,c,lens,window,sinks", [
    (1, 16, 1, [0], 1, None, 1, 0), (1, 16, 1, [15], 1, None, 1, 0), (2, 16, 40, [500, 3], 7, [7, 0], 100, 17), (3, 128, 9, [1000, 0, 300], 1, [0, 1, 1], 1, 0),
    (2, 32, 3000, [90000, 60001], 5000, None, 777, 33), (1, 16, 5000, [79999], 1, None, 1, 100000), (4, 64, 2049, [131000, 5, 64 * 2049 - 3, 70000], 3, None, 1, 1),
    (1, 16, 2048, [32767], 1, None, 2 ** 31 - 1, 0), (2, 16, 4097, [65551, 65551], 1, None, 1, 0)])
@pytest.mark.parametrize("inplace", [False, True])
def test_slide(a2sf, B, ps, mp, past, c, lens, window, sinks, inplace):
    pages = B * mp + 2
    g = torch.Generator().manual_seed(2)
    table = torch.randperm(pages, generator=g)[: B * mp].view(B, mp).to(I32)
    table[torch.rand((B, mp), generator=g) < 0.3] = -1                  # some have left before
    table[torch.rand((B, mp), generator=g) < 0.05] = -77
    cache = a2sf.PagedCache(B, 1, 64, BF, ps, pages, mp, page_table=table.cuda())
    cache.past.copy_(torch.tensor(past)), cache.start.copy_(torch.tensor(past) + 1000)
    ls = [c] * B if lens is None else lens
    n = [p + x for p, x in zip(past, ls)]
    want, freed = slide_ref(table, n, ps, window, sinks)
    if inplace:                                                         # entries that left before stay what they are
        want = torch.where(table < 0, table, want)
    fr, fc = torch.full((B, mp), -5, dtype=I32, device="cuda"), torch.full((B,), -5, dtype=I32, device="cuda")
    to, po, so = (None, None, None) if inplace else (torch.full((B, mp), -6, dtype=I32, device="cuda"), *(torch.zeros(B, dtype=I32, device="cuda") for _ in range(2)))
    cache.a2sf_paged_slide(window, sinks, c, lens=None if lens is None else torch.tensor(lens, dtype=I32).cuda(), table_out=to, freed=fr, freed_count=fc,
                           past_out=po, start_out=so)
    got = cache.page_table if inplace else to
    assert torch.equal(got.cpu(), want)
    assert fc.tolist() == [len(x) for x in freed]
    for b in range(B):
        assert fr[b, : len(freed[b])].tolist() == freed[b] and bool((fr[b, len(freed[b]):] == -5).all())
    assert (cache.past if inplace else po).tolist() == n and (cache.start if inplace else so).tolist() == [p + 1000 + x for p, x in zip(past, ls)]
    if not inplace:
        assert torch.equal(cache.page_table.cpu(), table) and cache.past.tolist() == past
        cache.a2sf_paged_slide(window, sinks, c, lens=None if lens is None else torch.tensor(lens, dtype=I32).cuda())        # no lists
        assert cache.past.tolist() == n


def test_slide_reports_entries_that_are_no_pages(a2sf):
    cache = a2sf.PagedCache(2, 1, 64, BF, 16, 10, 4, page_table=torch.tensor([[1, 10, 2, 3], [4, 5, 6, 2 ** 31 - 1]], dtype=I32).cuda())
    cache.past.copy_(torch.tensor([50, 50]))
    fr, fc = torch.full((2, 4), -5, dtype=I32, device="cuda"), torch.zeros(2, dtype=I32, device="cuda")
    cache.a2sf_paged_slide(1, freed=fr, freed_count=fc)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_ERR_INVALID_ARG
    assert cache.page_table.tolist() == [[-1, -1, -1, 3], [-1, -1, -1, 2 ** 31 - 1]]
    assert fc.tolist() == [2, 3] and fr.tolist() == [[1, 2, -5, -5], [4, 5, 6, -5]]


# ---- how calls are made ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,H,c,past,window", [(BF, 2, 1, 300, 100), (BF, 3, 4, 9000, 3000), (HF, 12, 300, 4000, 900), (FP, 2, 20, 50, 30), (BF, 2, 40, 100, 64)])
def test_graph_replay_and_other_stream(a2sf, dtype, H, c, past, window):
    """A captured step replayed with other lengths and inputs in the same tensors equals calls made one by one."""
    B, G, d = 2, 2, 128
    plan = a2sf.a2sf_rotary_axes_plan_init([d // 4, d // 4], a2sf.a2sf_rotary_plan_init(d), cycle=True)
    g = torch.Generator().manual_seed(21)
    steps = [[torch.randn((B, h, c, d), generator=g).to(dtype).cuda() for h in (H * G, H, H)] + [torch.randint(0, 99, (2, B, c), generator=g).to(I32).cuda()] for _ in range(3)]
    a, b = (pu.make_cache(a2sf, B, H, G, d, dtype, 32, [past, past // 3], 4 * c, seed=6) for _ in range(2))
    lens = [torch.tensor(x, dtype=I32).cuda() for x in ([c, c], [c, max(1, c // 2)], [0, c])]

    def step(cache, q, k, v, pos, L, out, lse):
        qr = cache.a2sf_paged_append_axes(k, v, pos, plan, lens=L, q=q)
        cache.a2sf_paged_attend_window(qr, window, 5, lens=L, out=out, lse=lse)
        cache.a2sf_paged_slide(window, 5, c, lens=L)

    want = []
    for (q, k, v, pos), L in zip(steps, lens):
        out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:3], 3.0, device="cuda")
        step(a, q, k, v, pos, L, out, lse)
        want.append((out, lse))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    inputs, L = [x.clone() for x in steps[0]], lens[0].clone()
    out, lse = torch.full_like(inputs[0], 3.0), torch.full(inputs[0].shape[:3], 3.0, device="cuda")
    state = [x.clone() for x in (b.page_table, b.past, b.start)]
    with torch.cuda.stream(side):
        step(b, *inputs, L, out, lse)                             # loads what a first call loads
        for x, y in zip((b.page_table, b.past, b.start), state):
            x.copy_(y)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(b, *inputs, L, out, lse)
        for x, y in zip((b.page_table, b.past, b.start), state):
            x.copy_(y)
        for new, ln, (o, z) in zip(steps, lens, want):
            for x, y in zip(inputs, new):
                x.copy_(y)
            L.copy_(ln)
            out.fill_(3.0), lse.fill_(3.0)
            graph.replay()
            side.synchronize()
            assert torch.equal(out, o) and torch.equal(lse, z)
    for name in ("page_table", "past", "start"):
        assert torch.equal(getattr(a, name), getattr(b, name))


def test_calls_on_two_streams_at_once(a2sf):
    B, H, G, d = 2, 4, 2, 128
    g = torch.Generator().manual_seed(31)
    data = [[torch.randn((B, h, c, d), generator=g).to(BF).cuda() for h in (H * G, H, H)] for c in (300, 1, 40, 1, 200, 3)]

    def run(cache, stream, results):
        for q, k, v in data:
            with torch.cuda.stream(stream):
                cache.a2sf_paged_append(k, v)
                results.append(cache.a2sf_paged_attend_window(q, 120, 9))
                cache.a2sf_paged_slide(120, 9, q.shape[2])
            yield

    caches = [pu.make_cache(a2sf, B, H, G, d, BF, 32, [100, 7], 600, seed=6) for _ in range(3)]
    torch.cuda.synchronize()
    alone, one, two = [], [], []
    for _ in run(caches[0], torch.cuda.current_stream(), alone):
        pass
    torch.cuda.synchronize()
    for _ in zip(run(caches[1], torch.cuda.Stream(), one), run(caches[2], torch.cuda.Stream(), two)):
        pass
    torch.cuda.synchronize()
    for a, b, c in zip(alone, one, two):
        for x, y, z in zip(a, b, c):
            assert torch.equal(x, y) and torch.equal(x, z)


def test_a_call_on_a_given_stream_allocates_there(a2sf):
    B, H, d, c = 2, 8, 128, 200
    g = torch.Generator().manual_seed(13)
    q, k, v = (torch.randn((B, H, c, d), generator=g).to(BF).cuda() for _ in range(3))
    cache = pu.make_cache(a2sf, B, H, 1, d, BF, 64, [3000, 2000], c, seed=6)
    cache.a2sf_paged_append(k, v)
    want = cache.a2sf_paged_attend_window(q, 1500, 4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, lse = cache.a2sf_paged_attend_window(q, 1500, 4, stream=side)
    for _ in range(20):                                 # would land in the workspace, were it the current stream's
        torch.full((cache.attend_window_workspace_bytes(c, 1500, 4) // 4,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_the_largest_batch_with_mostly_empty_sequences(a2sf):
    B = 1024
    past, lens = [0] * B, [0] * B
    for b, (p, n) in {0: (5, 1), 17: (100, 1), 500: (0, 1), 1023: (33, 1)}.items():
        past[b], lens[b] = p, n
    check_window(a2sf, (B, 1, 1, 64, BF, 16, past, 1, lens, 20, 3, "bhnd", 0.0))
    lens = [20 * n for n in lens]
    check_window(a2sf, (B, 1, 1, 64, HF, 16, past, 20, lens, 20, 3, "bhnd", 0.0))


@pytest.mark.parametrize("B,H,c,dtype,lens", [(300, 2, 140, BF, [140, 0, 17, 139, 1]), (1024, 1, 300, HF, [0] * 60 + [300, 0, 129, 1])])
def test_many_sequences_in_large_chunks(a2sf, B, H, c, dtype, lens):
    """The list of items over hundreds of sequences, most of them short or empty."""
    check_window(a2sf, (B, H, 1, 64, dtype, 16, [b % 13 for b in range(B)], c, [lens[b % len(lens)] for b in range(B)], 50, 3, "bhnd", 0.0))


@pytest.mark.parametrize("dtype,H,c", [(FP, 2, 3), (BF, 2, 1), (HF, 12, 300), (BF, 2, 40), (BF, 2, 4)])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "pages", "past", "negative", "length"])
def test_bad_pages_and_lengths_are_reported_and_not_followed(a2sf, dtype, H, c, bad):
    """A page in the window that is none, lengths outside the table: an error status, no access outside the pool, and the other sequence's results."""
    G, d, ps, window = 2, 64, 16, 60
    cache = pu.make_cache(a2sf, 2, H, G, d, dtype, ps, [90, 70], c, seed=6, garbage=0.0)
    g = torch.Generator().manual_seed(22)
    q, k, v = (torch.randn((2, h, c, d), generator=g).to(dtype).cuda() for h in (H * G, H, H))
    cache.a2sf_paged_append(k, v)
    want = cache.a2sf_paged_attend_window(q, window, 2)
    lens = None
    if bad == "past":
        cache.past[0] = 2 ** 31 - 1
    elif bad == "negative":
        cache.past[0] = -5
    elif bad == "length":
        lens = torch.tensor([-3, c], dtype=I32).cuda()
    else:
        cache.page_table[0, 4] = cache.num_pages if bad == "pages" else bad
    got = cache.a2sf_paged_attend_window(q, window, 2, lens=lens)
    torch.cuda.synchronize()
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_ERR_INVALID_ARG
    assert torch.equal(got[0][1], want[0][1]) and torch.equal(got[1][1], want[1][1])


@pytest.mark.parametrize("dtype,H,c", [(BF, 1, 1), (HF, 8, 200), (FP, 1, 20)])
def test_a_call_far_inside_a_large_pool_is_the_same(a2sf, dtype, H, c):
    """Pages behind 2^32 bytes (and elements) of the pool, and a page table whose slots are far from the first: the same bits."""
    d, ps, past, window, sinks = 128, 128, 3000, 700, 130
    esize = torch.finfo(dtype).bits // 8
    far_pages = (2 ** 32 + 2 ** 28) // (H * ps * d * esize)
    mp = -(-(past + c) // ps)
    g = torch.Generator().manual_seed(23)
    q, k, v = (torch.randn((1, H, n, d), generator=g).to(dtype).cuda() for n in (c, past + c, past + c))
    results = []
    for first in (0, far_pages):
        cache = a2sf.PagedCache(1, H, d, dtype, ps, first + mp, mp)
        cache.page_table.copy_((first + torch.randperm(mp, generator=torch.Generator().manual_seed(1))).view(1, -1))
        cache.a2sf_paged_append(k, v)
        cache.past.fill_(past)
        results.append([x.cpu() for x in cache.a2sf_paged_attend_window(q, window, sinks)])
        del cache
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_inputs_whose_rows_overlap_or_lie_apart(a2sf):
    g = torch.Generator().manual_seed(14)
    H, n, d = 4, 20, 64
    base = torch.randn((H + n, d), generator=g).to(BF).cuda()
    for x in (base.as_strided((1, H, n, d), (0, d, d, 1)), torch.randn((1, n, 3 * H, d), generator=g).to(BF).cuda().transpose(1, 2)[:, ::3]):
        flat = x.contiguous()
        a = pu.make_cache(a2sf, 1, H, 1, d, BF, 16, [40], n, seed=6)
        a.a2sf_paged_append(flat, flat)
        for got, want in zip(a.a2sf_paged_attend_window(x, 11, 2), a.a2sf_paged_attend_window(flat, 11, 2)):
            assert torch.equal(got, want)
