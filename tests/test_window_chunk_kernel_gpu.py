"""What the windowed attention promises, in calls that are large enough for its tcgen05 kernel: every test asserts that they take it,
and whether items were cut, in which case partial results go through the workspace."""
import math
import random

import pytest
import torch

import paged_util as pu
import test_window_gpu as tw
from window_forms import attend, tcgen05_bytes

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
BF, HF = torch.bfloat16, torch.float16
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


def check_rows(out, lse, K, V, q, past, window, sinks, scale, what):
    """Rows of one sequence and K/V head: out, lse [G][n](d) against K, V [L][d] and q [G][n][d] on the CPU."""
    o, z, size, logit, most, vmax = tw.window_ref(K.double(), V.double(), q.double(), past, window, sinks, scale)
    u, e = torch.finfo(out.dtype).eps / 2, (q.shape[-1] + 2) * F * logit
    under = 0.0 if out.dtype != HF else 2.0 ** -25 * most * vmax
    tw.close(out, o, u * o.abs() + (u + 2 * e + 2.0 ** -20 + most * F) * size + under, f"out {what}")
    tw.close(lse, z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), f"lse {what}")


# B, H, G, d, dtype, past of the first sequence, c, window, sinks, whether items are cut
CALLS = {"whole": (2, 24, 2, 64, HF, 90, 300, 60, 2, False), "whole, 128": (2, 12, 1, 128, BF, 500, 300, 450, 130, False),
         "cut": (1, 4, 4, 128, HF, 5000, 64, 4096, 4, True), "cut, two": (2, 6, 1, 64, BF, 9000, 500, 3000, 0, True)}


def made(a2sf, name, seed=6, garbage=0.0):
    B, H, G, d, dtype, past, c, window, sinks, cut = CALLS[name]
    cache = pu.make_cache(a2sf, B, H, G, d, dtype, 64 if past > 1000 else 16, [past, past * 3 // 4][:B], c, seed=seed, garbage=garbage)
    g = torch.Generator().manual_seed(22)
    q, k, v = (torch.randn((B, h, c, d), generator=g).to(dtype).cuda() for h in (H * G, H, H))
    cache.a2sf_paged_append(k, v)
    return cache, q, "tcgen05, cut" if cut else "tcgen05"


@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "pages"])
@pytest.mark.parametrize("name", CALLS)
def test_bad_pages_are_reported_and_not_followed(a2sf, name, bad):
    """A page in the first sequence's window that is none: an error status and the other sequence's results; rows that do not see it
    are as they were."""
    cache, q, form = made(a2sf, name)
    B, H, G, d, dtype, past, c, window, sinks, _ = CALLS[name]
    out, lse, got = attend(a2sf, cache, q, window, sinks)
    assert got == form
    at = (past + c - 1 - window // 2) // cache.page_size
    good = int(cache.page_table[0, at])
    cache.page_table[0, at] = cache.num_pages if bad == "pages" else bad
    out2, lse2, got = attend(a2sf, cache, q, window, sinks)
    assert got == form
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_ERR_INVALID_ARG
    if B > 1:
        assert torch.equal(out[1], out2[1]) and torch.equal(lse[1], lse2[1])
    p = past + torch.arange(c)
    first, last = at * cache.page_size, (at + 1) * cache.page_size - 1
    apart = ((p < first) | (p - window >= last)) & (first >= sinks)
    rows = apart.cuda()
    # a warp whose other rows saw the page may have moved its references: the same up to rounding
    u = torch.finfo(dtype).eps / 2
    assert float((out[0][:, rows].float() - out2[0][:, rows].float()).abs().max() if apart.any() else 0.0) <= 4 * u * float(cache.v_pages.float().abs().max())
    cache.page_table[0, at] = good
    out3, lse3, _ = attend(a2sf, cache, q, window, sinks)
    assert torch.equal(out, out3) and torch.equal(lse, lse3)


@pytest.mark.parametrize("bad", ["past", "negative", "length"])
@pytest.mark.parametrize("name", ["whole", "whole, 128", "cut, two"])
def test_bad_lengths_are_reported_and_not_followed(a2sf, name, bad):
    cache, q, form = made(a2sf, name)
    B, H, G, d, dtype, past, c, window, sinks, _ = CALLS[name]
    want, z, got = attend(a2sf, cache, q, window, sinks)
    assert got == form
    lens = None
    if bad == "past":
        cache.past[0] = 2 ** 31 - 1
    elif bad == "negative":
        cache.past[0] = -5
    else:
        lens = torch.tensor([-3, c], dtype=I32).cuda()
    out, lse, _ = attend(a2sf, cache, q, window, sinks, lens=lens)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_ERR_INVALID_ARG
    # where the cuts lie depends on the other sequences' lengths: the same up to the storage type's rounding and the order of sums
    K, V = (pu.slots(cache, getattr(cache, x).cpu(), 1, past * 3 // 4 + c) for x in ("k_pages", "v_pages"))
    for h in (0, H - 1):
        check_rows(out[1, h * G:(h + 1) * G], lse[1, h * G:(h + 1) * G], K[h], V[h], q[1, h * G:(h + 1) * G].cpu(), past * 3 // 4, window, sinks, 1 / math.sqrt(d), h)
    if form == "tcgen05":
        assert torch.equal(out[1], want[1]) and torch.equal(lse[1], z[1])


@pytest.mark.parametrize("H,c,past,window,sinks,form", [(8, 400, 3000, 700, 130, "tcgen05"), (4, 256, 6000, 4000, 4, "tcgen05, cut")])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_call_far_inside_a_large_pool_is_the_same(a2sf, dtype, H, c, past, window, sinks, form):
    """Pages behind 2^32 bytes of the pool: the same bits."""
    d, ps = 128, 128
    far_pages = (2 ** 32 + 2 ** 28) // (H * ps * d * 2)
    mp = -(-(past + c) // ps)
    g = torch.Generator().manual_seed(23)
    q, k, v = (torch.randn((1, H, n, d), generator=g).to(dtype).cuda() for n in (c, past + c, past + c))
    results = []
    for first in (0, far_pages):
        cache = a2sf.PagedCache(1, H, d, dtype, ps, first + mp, mp)
        cache.page_table.copy_((first + torch.randperm(mp, generator=torch.Generator().manual_seed(1))).view(1, -1))
        cache.a2sf_paged_append(k, v)
        cache.past.fill_(past)
        out, lse, got = attend(a2sf, cache, q, window, sinks)
        assert got == form
        results.append((out.cpu(), lse.cpu()))
        del cache
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_calls_on_two_streams_at_once(a2sf):
    """Whole items and cut ones, whose partial results lie in workspaces that the calls allocate, in steps on two streams."""
    B, H, G, d, window, sinks = 1, 8, 4, 128, 3000, 9
    g = torch.Generator().manual_seed(31)
    chunks = (400, 64, 200, 1, 64, 300)
    data = [[torch.randn((B, h, c, d), generator=g).to(BF).cuda() for h in (H * G, H, H)] for c in chunks]
    caches = [pu.make_cache(a2sf, B, H, G, d, BF, 32, [4000], sum(chunks), seed=6) for _ in range(3)]
    forms, alone = [], []
    for q, k, v in data:
        caches[0].a2sf_paged_append(k, v)
        out, lse, form = attend(a2sf, caches[0], q, window, sinks)
        alone.append((out, lse)), forms.append(form)
        caches[0].a2sf_paged_slide(window, sinks, q.shape[2])
    assert forms.count("tcgen05, cut") >= 4, forms
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    results = [[], []]
    for q, k, v in data:
        for s, cache, res in zip(streams, caches[1:], results):
            with torch.cuda.stream(s):
                cache.a2sf_paged_append(k, v)
                res.append(cache.a2sf_paged_attend_window(q, window, sinks))
                cache.a2sf_paged_slide(window, sinks, q.shape[2])
    torch.cuda.synchronize()
    for want, one, two in zip(alone, *results):
        for x, y, z in zip(want, one, two):
            assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.parametrize("H,c,past,window,form", [(30, 300, 500, 140, "tcgen05"), (4, 256, 6000, 4000, "tcgen05, cut")])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_rows_whose_logits_are_all_far_below_zero(a2sf, dtype, H, c, past, window, form):
    """All logits -200 (log2 units -288) in most slots, 0 in a few: a row whose first visible tile holds only low ones keeps them, and a
    piece that holds only low ones weighs nothing beside one that does not."""
    d, ps = 128, 64
    n = past + c
    pages = -(-n // ps)
    cache = a2sf.PagedCache(1, H, d, dtype, ps, pages, pages, scale=1.0)
    cache.page_table.copy_(torch.arange(pages).view(1, -1))
    k, v = torch.zeros((1, H, n, d), dtype=dtype), torch.randn((1, H, n, d), generator=torch.Generator().manual_seed(3)).to(dtype)
    k[..., 0] = -200.0
    k[0, :, 40, 0] = 0.0
    k[0, :, past - window + c // 2, 0] = 0.0                   # in the window of the first rows only
    k[0, :, past - window // 3, 0] = 0.0
    q = torch.zeros((1, H, c, d), dtype=dtype)
    q[..., 0] = 1
    cache.a2sf_paged_append(k.cuda(), v.cuda())
    cache.past.fill_(past)
    for sinks in (0, 3, 41):
        out, lse, got = attend(a2sf, cache, q.cuda(), window, sinks)
        assert got == form
        for h in (0, H - 1):
            o, z, size, logit, most, vmax = tw.window_ref(k[0, h].double(), v[0, h].double(), q[0, h:h + 1].double(), past, window, sinks, 1.0)
            u, e = torch.finfo(dtype).eps / 2, (d + 2) * F * 200
            under = 0.0 if dtype != HF else 2.0 ** -25 * most * vmax
            tw.close(out[0, h:h + 1], o, u * o.abs() + (u + 2 * e + 2.0 ** -20 + most * F) * size + under, f"out {sinks}")
            tw.close(lse[0, h:h + 1], z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), f"lse {sinks}")


@pytest.mark.parametrize("dtype,G,d,H", [(BF, 1, 128, 12), (HF, 4, 64, 12)])
def test_steps_in_recycled_pages(a2sf, dtype, G, d, H):
    """Chunks from one small pool: append, attend, slide; freed pages are made NaN and given out again.  Every row equals attention over
    all tokens so far."""
    B, ps, window, sinks, chunks = 2, 16, 70, 20, (300, 320, 5, 300)
    n = sum(chunks)
    g = torch.Generator().manual_seed(17)
    q, k, v = (torch.randn((B, h, n, d), generator=g).to(dtype).cuda() for h in (H * G, H, H))
    free = list(range(B * (max(chunks) + window + sinks + 3 * ps) // ps + 4))
    random.Random(3).shuffle(free)
    cache = a2sf.PagedCache(B, H, d, dtype, ps, len(free), -(-n // ps), group=G)
    cache.k_pages.fill_(float("nan")), cache.v_pages.fill_(float("nan"))
    at, forms = 0, []
    for c in chunks:
        table = cache.page_table.cpu()
        for b in range(B):
            for e in range(at // ps, -(-(at + c) // ps)):
                if table[b, e] < 0:
                    table[b, e] = free.pop()
        cache.page_table.copy_(table)
        cache.a2sf_paged_append(k[:, :, at : at + c], v[:, :, at : at + c])
        out, lse, form = attend(a2sf, cache, q[:, :, at : at + c], window, sinks)
        forms.append(form)
        for b in range(B):
            for h in (0, 5, H - 1):
                rows = slice(h * G, (h + 1) * G)
                check_rows(out[b, rows], lse[b, rows], k[b, h, : at + c].cpu(), v[b, h, : at + c].cpu(), q[b, rows, at : at + c].cpu(), at, window, sinks,
                           1 / math.sqrt(d), f"{at} {b} {h}")
        freed, count = torch.full_like(cache.page_table, -9), torch.zeros(B, dtype=I32, device="cuda")
        cache.a2sf_paged_slide(window, sinks, c, freed=freed, freed_count=count)
        at += c
        for b in range(B):
            got = freed[b, : int(count[b])].tolist()
            free += got
            for page in got:
                cache.k_pages[page].fill_(float("nan")), cache.v_pages[page].fill_(float("nan"))
    assert forms.count("tcgen05") >= 3, forms


@pytest.mark.parametrize("seed", range(24))
def test_random_calls(a2sf, seed):
    """Drawn until the call is the tcgen05 kernel's, which the size of its workspace tells."""
    r = random.Random(2000 + seed)
    while True:
        B, H, G, d = r.choice([1, 2, 4]), r.choice([6, 10, 16, 30]), r.choice([1, 2, 3, 4, 5, 8]), r.choice([64, 128])
        c = int(2 ** r.uniform(5, 9.5)) // min(G, 3) + 1
        past = [int(2 ** r.uniform(0, 12.5)) - 1 for _ in range(B)]
        dtype, ps, window, sinks = r.choice([BF, HF]), r.choice([16, 32, 64, 128]), int(2 ** r.uniform(0, 12.5)), r.choice([0, 1, 4, 17, 130])
        if c * G <= 16 or B * H * G * c * (max(past) + c) > 4e7:      # what the 64-bit form takes
            continue
        probe = a2sf.PagedCache(B, H, d, dtype, ps, 1, -(-(max(past) + c) // ps), group=G)
        if probe.attend_window_workspace_bytes(c, window, sinks) == tcgen05_bytes(B, H, G, d, c):
            break
    lens = [r.choice([c, c, 0, r.randint(0, c)]) for _ in range(B)]
    tw.check_window(a2sf, (B, H, G, d, dtype, ps, past, c, lens, window, sinks, r.choice(["bhnd", "bnhd"]), r.choice([0.0, 0.2])), seed=seed + 700)


def test_a_captured_cut_call_replays_beside_an_eager_one(a2sf):
    """Two graphs and an eager call of the same shape, whose workspaces are their own, one after the other and on two streams."""
    cache, q, form = made(a2sf, "cut")
    window, sinks = CALLS["cut"][7:9]
    want, z, got = attend(a2sf, cache, q, window, sinks)
    assert got == form == "tcgen05, cut"
    qs = [q, q.flip(2).contiguous()]
    other = attend(a2sf, cache, qs[1], window, sinks)[:2]
    graphs, outs = [], []
    for x in qs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(cache.a2sf_paged_attend_window(x, window, sinks))
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        eager = cache.a2sf_paged_attend_window(q, window, sinks)
        torch.cuda.synchronize()
        for got, ref in ((outs[0], (want, z)), (outs[1], other), (eager, (want, z))):
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
