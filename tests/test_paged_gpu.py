"""Rotary positions and the cache in pages against plain 64-bit forms on a B200.

Tolerances count roundings.  u = torch.finfo(dtype).eps / 2 is the half step of the storage type, f = 2^-24 that
of fp32.  A logit is a sum of d products in fp32: off by at most (d + 2) f * sum|q k| * scale =: e.  A probability is
then off by 2 e + 2^-20 relatively (its own logit, its row's log-sum-exp, the exponential)."""
import math
import random

import pytest
import torch

import paged_util as pu

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


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


# ---- rotary ---------------------------------------------------------------------------------------------

ROT = [
    # B, H, n, d, dtype, r, interleaved, scaling, start, transpose, layout
    (1, 1, 1, 64, BF, 64, False, "none", 0, False, "bhnd"),
    (2, 5, 7, 128, BF, 128, False, "none", 3, False, "bhnd"),
    (2, 5, 7, 128, HF, 128, True, "linear", 1000003, False, "bnhd"),
    (3, 2, 33, 64, FP, 32, True, "ramp", 2000000000, True, "bhnd"),
    (1, 3, 65, 64, FP, 24, False, "ntk", 130000, False, "bnhd"),
    (2, 4, 19, 128, HF, 24, False, "bands", 99999, True, "bnhd"),
    (2, 3, 5, 64, BF, 2, False, "none", 77, False, "bhnd"),
    (2, 3, 5, 64, BF, 6, True, "none", 77, False, "bhnd"),
    (1, 40, 130, 128, BF, 36, False, "bands", 50000, False, "bhnd"),
    (4, 1, 257, 128, FP, 126, False, "none", 12345, False, "bhnd"),
    (2, 2, 9, 128, FP, 128, True, "ntk", 0, True, "bhnd"),
]


def _scaling(scaling):
    return dict(scaling=scaling, factor=1.0 if scaling == "none" else 8.0, original_length=4096, low=1.0,
                high=32.0 if scaling == "ramp" else 4.0)


@pytest.mark.parametrize("case", ROT, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_rotary(a2sf, case):
    B, H, n, d, dtype, r, il, scaling, start, transpose, layout = case
    g = torch.Generator().manual_seed(1)
    x = torch.randn((B, H, n, d) if layout == "bhnd" else (B, n, H, d), generator=g).to(dtype)
    x = x if layout == "bhnd" else x.transpose(1, 2)
    kw = _scaling(scaling)
    plan = a2sf.a2sf_rotary_plan_init(r, interleaved=il, **kw)
    freqs = pu.inv_freq(r, 10000.0, scaling, kw["factor"], 4096, kw["low"], kw["high"])
    mag = 0.1 * math.log(8.0) + 1 if scaling == "ramp" else 1.0
    starts = torch.tensor([start + 11 * b for b in range(B)], dtype=torch.int32)
    lens = torch.tensor([n if b == 0 else max(0, n - 4 * b) for b in range(B)], dtype=torch.int32)
    want = torch.stack([pu.rotate(x[b].double(), starts[b].long() + torch.arange(n), freqs, il, mag, transpose) for b in range(B)])
    xc = x.cuda() if layout == "bhnd" else x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    out = torch.full_like(xc, 9.0)
    got = a2sf.a2sf_rotary(plan, xc, out=out, start=starts.cuda(), lens=lens.cuda(), transpose=transpose)
    live = (torch.arange(n) < lens[:, None])[:, None, :, None]
    size = x.double().norm(dim=-1, keepdim=True) * mag            # no pair is longer than its row
    u = torch.finfo(dtype).eps / 2
    tol = u * want.abs() + size * (2e-7 + 4 * F)
    close(torch.where(live.cuda(), got, torch.zeros_like(got)), torch.where(live, want, torch.zeros_like(want)), tol, "rotary")
    assert bool((got == 9.0)[~live.cuda().expand_as(got)].all()), "rows past the length were written"
    assert bool((got.cpu()[..., r:] == x[..., r:])[live.expand_as(x)[..., r:]].all()), "elements past rotary_dim are copies"
    # in place, and by explicit positions: the same bits
    again = a2sf.a2sf_rotary(plan, xc, out=xc, positions=(starts[:, None] + torch.arange(n, dtype=torch.int32)).cuda(),
                             lens=lens.cuda(), transpose=transpose)
    assert again.data_ptr() == xc.data_ptr()
    assert torch.equal(again[live.cuda().expand_as(again)], got[live.cuda().expand_as(got)])


def test_rotary_gradient_by_differences_and_inverse(a2sf):
    plan = a2sf.a2sf_rotary_plan_init(64)
    g = torch.Generator().manual_seed(3)
    x, dy, e = (torch.randn((2, 3, 9, 64), generator=g).cuda() for _ in range(3))
    dx = a2sf.a2sf_rotary(plan, dy, transpose=True)
    # y is linear in x: <dy, y(x + h e) - y(x)> / h = <dx, e>, up to the rounding of the two forward passes
    h = 0.5
    diff = ((a2sf.a2sf_rotary(plan, x + h * e).double() - a2sf.a2sf_rotary(plan, x).double()) * dy.double()).sum() / h
    want = (dx.double() * e.double()).sum()
    tol = 8 * (2e-7 + 4 * F) * float((x.norm() + e.norm()) * dy.norm() / h)
    assert abs(float(diff - want)) <= tol
    back = a2sf.a2sf_rotary(plan, a2sf.a2sf_rotary(plan, x), transpose=True)
    assert float((back - x).abs().max()) <= 2 * (2e-7 + 4 * F) * float(x.norm(dim=-1).max())


# ---- append --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("B,H,G,d,dtype,ps,c,r,il,layout", [
    (1, 1, 1, 64, FP, 16, 1, 64, False, "bhnd"),
    (3, 2, 4, 128, BF, 32, 37, 128, False, "bnhd"),
    (2, 5, 3, 128, HF, 64, 130, 24, True, "bhnd"),
    (4, 3, 8, 64, HF, 128, 5, 20, False, "bnhd"),
    (2, 2, 2, 128, BF, 16, 17, 0, False, "bhnd"),
])
def test_append(a2sf, B, H, G, d, dtype, ps, c, r, il, layout):
    past = [(5 * b + 3) % 41 for b in range(B)]
    cache = pu.make_cache(a2sf, B, H, G, d, dtype, ps, past, c, seed=2)
    before = {x: getattr(cache, x).cpu().clone() for x in ("k_pages", "v_pages", "scores", "positions")}
    start = torch.tensor([1000 * b + 7 for b in range(B)], dtype=torch.int32)
    cache.start.copy_(start)
    g = torch.Generator().manual_seed(4)
    lens = torch.tensor([c if b == 0 else (c * (b + 1)) % (c + 1) for b in range(B)], dtype=torch.int32)

    def tensor(h):
        t = torch.randn((B, h, c, d), generator=g).to(dtype)
        return t, (t.cuda() if layout == "bhnd" else t.transpose(1, 2).contiguous().cuda().transpose(1, 2))

    (k, kc), (v, vc), (q, qc) = tensor(H), tensor(H), tensor(H * G)
    plan = a2sf.a2sf_rotary_plan_init(r, interleaved=il) if r else None
    freqs = pu.inv_freq(r) if r else []
    q_out = torch.full_like(qc, 5.0)
    got = cache.a2sf_paged_append(kc, vc, lens=lens.cuda(), q=qc if r else None, q_out=q_out if r else None, rotary=plan)
    after = {x: getattr(cache, x).cpu() for x in before}
    want = {x: t.clone().double() if t.is_floating_point() else t.clone() for x, t in before.items()}
    tol = {"k_pages": torch.zeros_like(want["k_pages"])}
    u = torch.finfo(dtype).eps / 2
    table = cache.page_table.cpu()
    for b in range(B):
        pos = start[b].long() + torch.arange(c)
        kr = pu.rotate(k[b].double(), pos, freqs, il)
        for t in range(int(lens[b])):
            pg, o = int(table[b, (past[b] + t) // ps]), (past[b] + t) % ps
            want["k_pages"][pg, :, o] = kr[:, t]
            tol["k_pages"][pg, :, o] = u * kr[:, t].abs() + k[b, :, t].double().norm(dim=-1, keepdim=True) * (2e-7 + 4 * F) * bool(r)
            want["v_pages"][pg, :, o] = v[b, :, t].double()
            want["scores"][pg, :, o] = 0
            want["positions"][pg, :, o] = int(pos[t])
        if r:
            n = int(lens[b])
            qr = pu.rotate(q[b].double(), pos, freqs, il)
            close(got[b, :, :n], qr[:, :n], u * qr[:, :n].abs() + q[b, :, :n].double().norm(dim=-1, keepdim=True) * (2e-7 + 4 * F), "q")
            assert bool((got[b, :, n:] == 5.0).all())
    garbage = torch.isnan(want["k_pages"])
    assert torch.equal(torch.isnan(after["k_pages"]), garbage), "slots outside the chunk were touched"
    close(torch.where(garbage.cuda(), torch.zeros_like(cache.k_pages), cache.k_pages), want["k_pages"].nan_to_num(0.0), tol["k_pages"], "keys")
    assert torch.equal(after["v_pages"].double().nan_to_num(7.0), want["v_pages"].nan_to_num(7.0))
    assert torch.equal(after["scores"].double().nan_to_num(7.0), want["scores"].nan_to_num(7.0))
    assert torch.equal(after["positions"], want["positions"])
    assert cache.past.tolist() == past


# ---- attend ----------------------------------------------------------------------------------------------

ATT = [
    # B, H, G, d, dtype, ps, past, c, lens, alpha, layout, scale
    (1, 1, 1, 64, FP, 16, [0], 1, None, 0.5, "bhnd", 0.0),                     # one token, nothing before it
    (2, 2, 1, 64, FP, 16, [0, 0], 129, None, 0.5, "bhnd", 0.0),
    (3, 2, 3, 128, FP, 32, [70, 0, 5], 33, [33, 0, 20], 0.9, "bnhd", 0.2),
    (2, 1, 8, 128, FP, 64, [1000, 33], 1, [1, 0], 1.0, "bhnd", 0.0),
    (2, 3, 5, 64, FP, 128, [200, 64], 70, [70, 69], 0.0, "bnhd", 0.0),
    (4, 3, 1, 128, BF, 16, [204, 0, 63, 64], 1, None, 0.3, "bhnd", 0.0),       # few rows
    (5, 2, 1, 128, BF, 64, [130, 7, 500, 0, 1], 1, [1, 0, 1, 1, 1], 0.5, "bhnd", 0.0),
    (2, 2, 4, 128, HF, 64, [1999, 17], 4, [4, 3], 0.9, "bnhd", 0.0),
    (2, 2, 8, 64, HF, 32, [333, 100], 1, None, 1.0, "bhnd", 0.0),
    (1, 3, 8, 128, BF, 128, [640], 2, None, 0.0, "bhnd", 0.3),
    (3, 1, 5, 64, BF, 16, [37, 0, 90], 3, [3, 2, 0], 0.7, "bnhd", 0.0),
    (1, 2, 3, 128, HF, 16, [9000], 5, None, 0.99, "bhnd", 0.0),                # one long sequence
    (2, 1, 2, 64, BF, 64, [4096, 4095], 1, None, 0.5, "bhnd", 0.0),
    (1, 1, 1, 128, HF, 16, [0], 17, None, 0.5, "bhnd", 0.0),                   # many rows
    (2, 2, 1, 128, BF, 64, [0, 0], 128, [128, 127], 0.9, "bhnd", 0.0),
    (2, 2, 4, 128, HF, 32, [0, 300], 200, [200, 77], 1.0, "bnhd", 0.0),
    (3, 1, 5, 128, BF, 16, [511, 0, 129], 100, [100, 0, 51], 0.5, "bhnd", 0.0),
    (1, 2, 8, 64, HF, 128, [1000], 129, None, 0.9, "bhnd", 0.0),
    (2, 1, 3, 64, BF, 64, [0, 77], 300, [300, 1], 1.0, "bnhd", 0.25),
    (1, 1, 7, 128, BF, 16, [2500], 41, None, 0.0, "bhnd", 0.0),
    (2, 3, 1, 128, HF, 128, [640, 1], 513, [513, 512], 0.999, "bhnd", 0.0),
]


def check_attend(a2sf, case, seed=5, garbage=float("nan"), gain=1.0, room=0):
    B, H, G, d, dtype, ps, past, c, lens, alpha, layout, scale = case
    lens = [c] * B if lens is None else lens
    cache = pu.make_cache(a2sf, B, H, G, d, dtype, ps, past, max(c, room), seed=seed, scale=scale, garbage=garbage)
    g = torch.Generator().manual_seed(seed + 1)

    def tensor(h, k=1.0):
        t = (torch.randn((B, h, c, d), generator=g) * k).to(dtype)
        return t, (t.cuda() if layout == "bhnd" else t.transpose(1, 2).contiguous().cuda().transpose(1, 2))

    (k, kc), (v, vc), (q, qc) = tensor(H), tensor(H), tensor(H * G, gain)
    L = torch.tensor(lens, dtype=torch.int32).cuda()
    cache.a2sf_paged_append(kc, vc, lens=L)
    old = cache.scores.cpu().clone()
    pool_k, pool_v = cache.k_pages.cpu().double(), cache.v_pages.cpu().double()
    out, lse = torch.full_like(qc, 3.0), torch.full((B, H * G, c), 3.0, device="cuda")
    # the binding's torch: in the debug sweep it puts guard words around the workspace
    cache.a2sf_paged_attend(qc, alpha, lens=L, out=out, lse=lse, workspace=a2sf.torch.empty(
        (cache.attend_workspace_bytes(c),), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    sc = scale or 1 / math.sqrt(d)
    u = torch.finfo(dtype).eps / 2
    new, seen = cache.scores.cpu(), torch.zeros_like(old, dtype=torch.bool)
    for b in range(B):
        n, Lb = lens[b], past[b] + lens[b]
        assert bool((out[b, :, n:] == 3.0).all()) and bool((lse[b, :, n:] == 3.0).all()), "rows past the length were written"
        if n == 0:
            continue
        K, V, S, S1 = (pu.slots(cache, x, b, Lb) for x in (pool_k, pool_v, old.double(), new))
        t, j = cache.page_table.cpu()[b].long(), torch.arange(Lb)
        seen[t[j // ps], :, j % ps] = True
        for h in range(H):
            o, z, s, size, logit = pu.attend_ref(K[h], V[h], q[b, h * G:(h + 1) * G, :n].double(), S[h], past[b], alpha, sc)
            e = (d + 2) * F * logit
            rel = 2 * e + 2.0 ** -20
            # out: its own rounding, a probability's rounding to the storage type (fp16: 2^-25 absolutely below its
            # normal range, against a row sum of at least 1 at a scale of at most 2^8), the probability's own error
            under = 0.0 if dtype != HF else 2.0 ** -25 * Lb * float(V[h].abs().max())
            close(out[b, h * G:(h + 1) * G, :n], o, u * o.abs() + (u + rel + Lb * F) * size + under, f"out {b} {h}")
            close(lse[b, h * G:(h + 1) * G, :n], z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), f"lse {b} {h}")
            # scores: a weight's exponent is at most 150 with two roundings; the sums and the decayed old score
            close(S1[h], s, s * (rel + 150 * 2 * F + (n * G + 4) * F) + 1e-37, f"scores {b} {h}")
    assert torch.equal(new[~seen].nan_to_num(7.0), old[~seen].nan_to_num(7.0)), "scores outside the sequences were touched"
    return cache, qc, L, out, lse, old


@pytest.mark.parametrize("case", ATT, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "") for x in c))
def test_attend(a2sf, case):
    cache, qc, L, out, lse, old = check_attend(a2sf, case)
    # the same call again: the same bits; without scores: the same outputs and untouched scores
    cache.scores.copy_(old.cuda())
    out2, lse2 = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
    cache.a2sf_paged_attend(qc, case[9], lens=L, out=out2, lse=lse2)
    first = cache.scores.clone()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    cache.scores.copy_(old.cuda())
    cache.a2sf_paged_attend(qc, case[9], lens=L, out=out2, lse=lse2, scores=False)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    assert torch.equal(cache.scores.cpu().nan_to_num(7.0), old.nan_to_num(7.0))
    cache.a2sf_paged_attend(qc, case[9], lens=L, out=out2, lse=lse2)
    assert torch.equal(cache.scores.nan_to_num(7.0), first.nan_to_num(7.0))


@pytest.mark.parametrize("seed", range(40))
def test_attend_random_cases(a2sf, seed):
    check_attend(a2sf, random_attend(random.Random(seed)), seed=seed + 100)


def random_attend(r):
    B, H, G = r.choice([1, 1, 2, 3, 6]), r.choice([1, 2, 3]), r.choice([1, 1, 2, 3, 4, 5, 6, 7, 8])
    c = r.choice([1, 1, 2, 16 // G, 16 // G + 1, int(2 ** r.uniform(1, 9)), 128 // G, 256 // G + 1])
    past = [int(2 ** r.uniform(0, 10)) - 1 if r.random() < 0.9 else 0 for _ in range(B)]
    lens = [r.choice([c, c, c, 0, r.randint(0, c)]) for _ in range(B)]
    return (B, H, G, r.choice([64, 128]), r.choice([FP, BF, BF, HF]), r.choice([16, 32, 64, 128]), past, max(1, c), lens,
            r.choice([0.0, 0.3, 0.5, 0.9, 0.99, 1.0]), r.choice(["bhnd", "bnhd"]), r.choice([0.0, 0.0, 0.2]))


@pytest.mark.parametrize("dtype,c,past", [(BF, 1, 600), (HF, 1, 600), (FP, 1, 100), (BF, 150, 200), (HF, 150, 200), (HF, 4, 300)])
def test_attend_large_logits_and_late_maximum(a2sf, dtype, c, past):
    """Queries 12 times the usual size: logits of +-100, rows that one key takes whole, maxima that come late."""
    check_attend(a2sf, (1, 2, 2, 128, dtype, 32, [past], c, None, 0.9, "bhnd", 0.0), seed=9, gain=12.0)


@pytest.mark.parametrize("dtype,G,c,past", [(BF, 1, 1, 77), (HF, 4, 1, 200), (BF, 4, 40, 33), (FP, 1, 20, 30), (HF, 2, 150, 0)])
def test_attend_infinities_behind_the_sequence(a2sf, dtype, G, c, past):
    check_attend(a2sf, (2, 1, G, 128, dtype, 64, [past, 0], c, None, 0.5, "bhnd", 0.0), seed=11, garbage=float("inf"))


@pytest.mark.parametrize("dtype,chunks", [(FP, [40, 1, 29]), (BF, [1, 64, 5, 140, 2]), (HF, [200, 10, 1, 1])])
def test_chunks_of_a_prompt_give_the_scores_of_the_whole(a2sf, dtype, chunks):
    """append + attend over any split of a prompt equals the dense prefill of the library, scores and outputs."""
    B, H, d, n, alpha = 2, 3, 128, sum(chunks), 0.9
    g = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn((B, H, n, d), generator=g).to(dtype).cuda() for _ in range(3))
    p = a2sf.make_params(B, H, d, dtype, n, n, alpha)
    out, scores, _, lse = a2sf.a2sf_prefill(p, q, k, v)
    cache = a2sf.PagedCache(B, H, d, dtype, 16, 64, 30)
    cache.page_table.copy_(torch.randperm(64, generator=g)[:60].view(2, 30).to(torch.int32))
    at = 0
    for c in chunks:
        part = slice(at, at + c)
        cache.a2sf_paged_append(k[:, :, part], v[:, :, part])
        o, z = cache.a2sf_paged_attend(q[:, :, part], alpha)
        u = torch.finfo(dtype).eps / 2
        assert float((o.float() - out[:, :, part].float()).abs().max()) <= 4 * u * float(v.abs().max()) + 1e-5
        assert float((z - lse[:, :, part]).abs().max()) <= 2e-5
        cache.a2sf_paged_evict(n, 0, c)
        at += c
    assert cache.past.tolist() == [n] * B and cache.start.tolist() == [n] * B
    got = torch.stack([pu.slots(cache, cache.scores.cpu(), b, n) for b in range(B)])
    assert torch.allclose(got, scores.cpu(), rtol=1e-4, atol=1e-34)
    pos = torch.stack([pu.slots(cache, cache.positions.cpu(), b, n) for b in range(B)])
    assert torch.equal(pos, torch.arange(n, dtype=torch.int32).expand(B, H, n))


# ---- evict -----------------------------------------------------------------------------------------------

EVI = [
    # B, H, d, dtype, ps, past, c, budget, recent, fresh, scores
    (1, 1, 64, FP, 16, [0], 1, 1, 0, False, "rand"),
    (2, 3, 128, BF, 32, [100, 20], 5, 40, 16, False, "rand"),
    (2, 3, 128, BF, 32, [100, 20], 5, 40, 16, True, "rand"),
    (3, 2, 64, HF, 16, [333, 0, 64], 1, 64, 0, False, "zeros"),
    (3, 2, 64, HF, 16, [333, 0, 64], 1, 64, 64, True, "zeros"),
    (1, 2, 128, FP, 64, [1500], 7, 700, 350, False, "ties"),
    (1, 2, 128, FP, 64, [1500], 7, 1, 1, True, "ties"),
    (2, 1, 64, BF, 128, [2100, 1000], 1, 2000, 10, False, "signed"),
    (1, 1, 128, HF, 16, [20000], 3, 5000, 100, False, "rand"),
    (1, 2, 64, BF, 16, [20000], 1, 600, 599, True, "ties"),
    (2, 2, 64, BF, 16, [50, 60], 4, 100000, 7, False, "rand"),
    (1, 1, 64, BF, 128, [40000], 1, 30000, 100, False, "ties"),
    (1, 1, 64, HF, 128, [40000], 9, 9000, 1000, True, "rand"),
]


def check_evict(a2sf, case, seed=3):
    B, H, d, dtype, ps, past, c, budget, recent, fresh, kind = case
    n = [p + c for p in past]
    cache = pu.make_cache(a2sf, B, H, 1, d, dtype, ps, n, 0, seed=seed)      # the chunk is in place already
    cache.past.copy_(torch.tensor(past, dtype=torch.int32))
    start = [p + 1000 for p in past]
    cache.start.copy_(torch.tensor(start, dtype=torch.int32))
    g = torch.Generator().manual_seed(seed + 5)
    sc = torch.rand(cache.scores.shape, generator=g)
    if kind == "zeros":
        sc.zero_()
    elif kind == "ties":
        sc = (sc * 4).floor()
    elif kind == "signed":
        sc = torch.where(sc < 0.2, torch.full_like(sc, float("inf")), torch.where(sc > 0.9, -0.0 * sc, sc - 0.5))
        sc[sc.abs() < 0.01] = float("nan")
    cache.scores.copy_(sc)
    # positions: in no order, every head its own, up to the newest
    table = cache.page_table.cpu().long()
    for b in range(B):
        for h in range(H):
            pos = torch.randperm(n[b] + 1000, generator=g)[: n[b]].to(torch.int32)
            j = torch.arange(n[b])
            cache.positions[table[b, j // ps], h, j % ps] = pos.cuda()
    before = {x: getattr(cache, x).cpu().clone() for x in ("k_pages", "v_pages", "scores", "positions")}
    want = {x: t.clone() for x, t in before.items()}
    dst = None
    if fresh:
        spare = -(-budget // ps)
        extra = {x: torch.full((B * spare,) + t.shape[1:], 1, dtype=t.dtype) for x, t in want.items()}
        base = want["scores"].shape[0]
        want = {x: torch.cat([t, extra[x]]) for x, t in want.items()}
        dst = (base + torch.randperm(B * spare, generator=g)).to(torch.int32).view(B, spare)
        cache = a2sf.PagedCache(B, H, d, dtype, ps, base + B * spare, cache.max_pages, page_table=cache.page_table, past=cache.past,
                                start=cache.start, **{x: t.cuda() for x, t in want.items()})
        before = {x: t.clone() for x, t in want.items()}
    for b in range(B):
        m = min(n[b], budget)
        for h in range(H):
            j = torch.arange(n[b])
            s = before["scores"][table[b, j // ps], h, j % ps].tolist()
            s = [math.nextafter(math.inf, 0) if x == math.inf else math.inf if x != x else x for x in s]    # NaN beyond infinity
            pos = before["positions"][table[b, j // ps], h, j % ps].tolist()
            stay = pu.evict_ref(s, pos, n[b], budget, start[b] + c - recent)
            if fresh:
                moves = list(zip(stay, range(m)))
            else:
                holes = sorted(set(range(m)) - set(stay))
                moves = list(zip([x for x in stay if x >= m], holes))
            to_table = dst[b].long() if fresh else table[b]
            for x in want:
                for f, t in moves:
                    want[x][to_table[t // ps], h, t % ps] = before[x][table[b, f // ps], h, f % ps]
    cache.a2sf_paged_evict(budget, recent, c, dst_table=None if dst is None else dst.cuda(), workspace=a2sf.torch.empty(
        (cache.evict_workspace_bytes(budget),), dtype=torch.uint8, device="cuda"))
    assert cache.past.tolist() == [min(x, budget) for x in n]
    assert cache.start.tolist() == [s + c for s in start]
    for x in want:
        got = getattr(cache, x).cpu()
        if got.is_floating_point():
            assert torch.equal(got.double().nan_to_num(1e9), want[x].double().nan_to_num(1e9)), x
        else:
            assert torch.equal(got, want[x]), x


@pytest.mark.parametrize("case", EVI, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "") for x in c))
def test_evict(a2sf, case):
    check_evict(a2sf, case)


@pytest.mark.parametrize("seed", range(24))
def test_evict_random_cases(a2sf, seed):
    check_evict(a2sf, random_evict(random.Random(seed)), seed=seed + 50)


def random_evict(r):
    B, H, c = r.choice([1, 2, 3, 5]), r.choice([1, 2, 3]), r.choice([1, 2, 7, 8, 9, 40])
    past = [int(2 ** r.uniform(0, 10.5)) - 1 for _ in range(B)]
    budget = max(1, r.choice([int((max(past) + c) * r.uniform(0.05, 1.1)), past[0]]))
    return (B, H, r.choice([64, 128]), r.choice([FP, BF, HF]), r.choice([16, 32, 64, 128]), past, c, budget, r.choice([0, budget // 2, budget]),
            r.random() < 0.5, r.choice(["rand", "zeros", "ties", "signed"]))


def test_evict_of_many_heads_moves_rows_in_the_searching_blocks(a2sf):
    """More heads than the device has SMs twice over: the other form of the kernel, in place and into fresh pages."""
    for fresh in (False, True):
        check_evict(a2sf, (7, 47, 64, BF, 16, [40, 3, 0, 25, 90, 64, 33], 3, 30, 10, fresh, "ties"), seed=17)


def test_evict_with_positions_given_twice_keeps_exactly_the_budget(a2sf):
    """More recent slots than the budget holds (a position twice): ranked among themselves, lower slots leave first."""
    for n, budget, recent in ((60, 20, 10), (60, 57, 10), (60, 52, 52)):
        cache = pu.make_cache(a2sf, 1, 1, 1, 64, FP, 16, [n], 0, seed=3)
        cache.scores.fill_(0.5)
        cache.positions.fill_(n - 1)
        cache.past.fill_(n - 1)
        cache.start.fill_(n - 1)
        first = pu.slots(cache, cache.k_pages.cpu(), 0, n)[0]
        cache.a2sf_paged_evict(budget, recent, 1)
        assert cache.past.item() == budget and cache.start.item() == n
        # slots 0 .. n - budget - 1 leave, the last ones take their places in order
        got = pu.slots(cache, cache.k_pages.cpu(), 0, budget)[0]
        stay = list(range(n - budget, n))
        holes = [j for j in range(budget) if j not in stay]
        want = first[:budget].clone()
        for hole, src in zip(holes, [j for j in stay if j >= budget]):
            want[hole] = first[src]
        assert torch.equal(got, want)


# ---- the whole step -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,G", [(BF, 1), (HF, 4), (FP, 2)])
def test_generation_steps_equal_the_slot_cache(a2sf, dtype, G):
    """append + attend + evict of single tokens is the generation step of the slot cache: same outputs, and the same
    tokens stay (compared while no two scores at the cut are closer than the two paths' rounding)."""
    B, H, d, n, M, R, T, alpha = 2, 2, 128, 96, 48, 16, 24, 0.9
    g = torch.Generator().manual_seed(21)
    q, k, v = (torch.randn((B, h, n + T, d), generator=g).to(dtype).cuda() for h in (H * G, H, H))
    p = a2sf.make_params(B, H, d, dtype, M, R, alpha)
    out, scores, kept, _ = a2sf.a2sf_prefill_group(p, G, q[:, :, :n].contiguous(), k[:, :, :n].contiguous(), v[:, :, :n].contiguous())
    old = a2sf.Cache(p)
    old.a2sf_cache_load(k[:, :, :n].contiguous(), v[:, :, :n].contiguous(), scores, kept)
    new = a2sf.PagedCache(B, H, d, dtype, 16, 20, 9, group=G)
    new.page_table.copy_(torch.randperm(18, generator=g).view(2, 9).to(torch.int32))
    new.a2sf_paged_append(k[:, :, :n], v[:, :, :n])
    new.a2sf_paged_attend(q[:, :, :n], alpha)
    new.a2sf_paged_evict(M, R, n)
    u = torch.finfo(dtype).eps / 2
    o1 = torch.empty((B, H * G, d), dtype=dtype, device="cuda")
    ev = torch.empty((B, H), dtype=torch.int32, device="cuda")
    for t in range(n, n + T):
        old.a2sf_decode_step_group(G, alpha, q[:, :, t].contiguous(), k[:, :, t].contiguous(), v[:, :, t].contiguous(), o1, ev)
        new.a2sf_paged_append(k[:, :, t:t + 1], v[:, :, t:t + 1])
        o2, _ = new.a2sf_paged_attend(q[:, :, t:t + 1], alpha)
        new.a2sf_paged_evict(M, R, 1)
        assert float((o1.float() - o2[:, :, 0].float()).abs().max()) <= 4 * u * float(v.abs().max()) + 1e-5
    st = old.a2sf_cache_export()
    pos = torch.stack([pu.slots(new, new.positions.cpu(), b, M) for b in range(B)])
    assert torch.equal(st["pos"].cpu().sort(-1).values, pos.sort(-1).values)
    a = torch.gather(st["scores"].cpu(), 2, st["pos"].cpu().argsort(-1))
    b = torch.gather(torch.stack([pu.slots(new, new.scores.cpu(), x, M) for x in range(B)]), 2, pos.argsort(-1))
    assert torch.allclose(a, b, rtol=2e-4, atol=1e-30)


@pytest.mark.parametrize("dtype,c,past", [(BF, 1, 300), (HF, 150, 40), (FP, 20, 50)])
def test_graph_replay_and_other_stream(a2sf, dtype, c, past):
    """A captured step, replayed on new inputs while lengths move on, equals direct calls on another stream."""
    B, H, G, d, M = 2, 2, 2, 128, past
    plan = a2sf.a2sf_rotary_plan_init(d)
    g = torch.Generator().manual_seed(2)
    ins = [[torch.randn((B, h, c, d), generator=g).to(dtype).cuda() for h in (H * G, H, H)] for _ in range(3)]
    a, b = (pu.make_cache(a2sf, B, H, G, d, dtype, 32, [past, past // 2], 2 * c, seed=6) for _ in range(2))

    def step(cache, q, k, v, q2, out, lse):
        # other kernels before, between and after the library's
        cache.a2sf_paged_append(k * 0.5, v.clone(), q=q, q_out=q2, rotary=plan)
        q2.mul_(2.0)
        cache.a2sf_paged_attend(q2, 0.9, out=out, lse=lse)
        cache.scores.mul_(0.75)
        cache.a2sf_paged_evict(M, 8, c)
        cache.start.add_(1)

    q, k, v = (x.clone() for x in ins[0])
    q2, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((B, H * G, c), device="cuda")
    warm = pu.make_cache(a2sf, B, H, G, d, dtype, 32, [past, past // 2], 2 * c, seed=6)
    step(warm, q, k, v, q2, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, q, k, v, q2, out, lse)
    side = torch.cuda.Stream()
    for x in ins:
        for dst, src in zip((q, k, v), x):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            r2, o2, z2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(lse)
            step(b, *x, r2, o2, z2)
        side.synchronize()
        assert torch.equal(out, o2) and torch.equal(lse, z2) and torch.equal(q2, r2)
        for name in ("k_pages", "v_pages", "scores", "positions", "past", "start"):
            assert torch.equal(getattr(a, name).double().nan_to_num(7.0), getattr(b, name).double().nan_to_num(7.0)), name


# ---- what the device finds out ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,c", [(FP, 3), (BF, 1), (HF, 150), (BF, 4)])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "pages", "past", "negative", "length"])
def test_bad_pages_and_lengths_are_reported_and_not_followed(a2sf, dtype, c, bad):
    cache = pu.make_cache(a2sf, 2, 2, 1, 128, dtype, 16, [40, 30], c, seed=4, garbage=0.0)
    lens = torch.full((2,), c, dtype=torch.int32, device="cuda")
    if bad == "past":
        cache.past[1] = cache.max_pages * 16 + 5
    elif bad == "negative":
        cache.past[1] = -3
    elif bad == "length":
        lens[1] = -4
    else:
        cache.page_table[1, :] = cache.num_pages if bad == "pages" else bad
    guard = {x: getattr(cache, x).clone() for x in ("v_pages", "positions")}
    x = torch.randn((2, 2, c, 128), device="cuda").to(dtype)
    plan = a2sf.a2sf_rotary_plan_init(128)
    for call in (lambda: cache.a2sf_paged_append(x, x, q=x, rotary=plan, lens=lens), lambda: cache.a2sf_paged_attend(x, 0.5, lens=lens),
                 lambda: cache.a2sf_paged_evict(20, 4, c, lens=lens, past_out=torch.empty_like(cache.past), start_out=torch.empty_like(cache.past))):
        call()
        assert a2sf.a2sf_last_device_status() == a2sf.A2SF_ERR_INVALID_ARG
        assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK
    # the other sequence's pages and the unused ones: only its own chunk was written
    own = cache.page_table[0].long()
    others = torch.ones(cache.num_pages, dtype=torch.bool, device="cuda")
    others[own] = False
    if bad not in ("past", "negative", "length"):
        assert torch.equal(cache.v_pages[others], guard["v_pages"][others])
        assert torch.equal(cache.positions[others], guard["positions"][others])


# ---- large and together ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,c", [(BF, 1), (HF, 130), (FP, 1)])
def test_rows_beyond_32_bit_offsets(a2sf, dtype, c):
    """Pages at the end of a pool of more than 2^31 elements give what the same pages give in a small pool."""
    H, d, ps, past = 8, 128, 128, 300
    pages = (2 ** 31) // (H * ps * d) + 40
    rows = torch.arange(past + c)
    far = (pages - 1 - torch.arange(4)).to(torch.int32).view(1, 4).cuda()
    near = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(5)
    k, v, q = (torch.randn((1, H, past, d), generator=g).to(dtype).cuda(), torch.randn((1, H, past, d), generator=g).to(dtype).cuda(),
               torch.randn((1, H, past, d), generator=g).to(dtype).cuda())
    plan = a2sf.a2sf_rotary_plan_init(d)
    results = []
    for n_pages, table in ((pages, far), (4, near)):
        cache = a2sf.PagedCache(1, H, d, dtype, ps, n_pages, 4, page_table=table)
        cache.a2sf_paged_append(k, v)
        cache.a2sf_paged_evict(past, 0, past)
        part = slice(0, c)
        q2 = cache.a2sf_paged_append(k[:, :, part], v[:, :, part], q=q[:, :, part], rotary=plan)
        out, lse = cache.a2sf_paged_attend(q2, 0.9)
        scores = pu.slots(cache, cache.scores.cpu(), 0, past + c)
        cache.a2sf_paged_evict(200, 50, c)
        t = cache.page_table[0].long()
        pool = [x[t].cpu() for x in (cache.k_pages, cache.v_pages, cache.positions)]
        results.append([out.cpu(), lse.cpu(), scores] + [x.transpose(1, 2).reshape(4 * ps, H, -1)[:200] for x in pool])
        del cache
    assert len(rows) == past + c
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_calls_on_two_streams_at_once(a2sf):
    """Chunks and tokens of two caches, issued alternately on two streams with no order between them."""
    B, H, G, d = 2, 4, 2, 128
    g = torch.Generator().manual_seed(31)
    data = [[torch.randn((B, h, c, d), generator=g).to(BF).cuda() for h in (H * G, H, H)] for c in (300, 1, 40, 1, 200, 3)]

    def run(cache, streams, results):
        for q, k, v in data:
            with torch.cuda.stream(streams):
                cache.a2sf_paged_append(k, v)
                results.append(cache.a2sf_paged_attend(q, 0.9))
                cache.a2sf_paged_evict(250, 30, q.shape[2])
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


def test_a_stream_given_and_inputs_from_another(a2sf):
    """The stream argument: work is queued there, behind what that stream waits for."""
    x = torch.zeros((1, 2, 5, 64), device="cuda")
    plan = a2sf.a2sf_rotary_plan_init(64)
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    big = torch.randn((4096, 4096), device="cuda")
    for _ in range(20):
        big = big @ big * 1e-4                      # keeps the current stream busy
    x.copy_(torch.ones_like(x))
    side.wait_stream(main)
    out = torch.zeros_like(x)
    side.wait_stream(main)
    a2sf.a2sf_rotary(plan, x, out=out, stream=side)
    main.wait_stream(side)
    want = pu.rotate(torch.ones((1, 2, 5, 64), dtype=torch.float64), torch.arange(5), pu.inv_freq(64))
    close(out, want, torch.full_like(want, 8 * (2e-7 + 4 * F)), "rotary on a side stream")


def test_the_largest_batch_with_mostly_empty_sequences(a2sf):
    B = 1024
    past = [0] * B
    lens = [0] * B
    for b, (p, n) in {0: (5, 1), 17: (100, 1), 500: (0, 1), 1023: (33, 1)}.items():
        past[b], lens[b] = p, n
    check_attend(a2sf, (B, 1, 1, 64, BF, 16, past, 1, lens, 0.5, "bhnd", 0.0))
    lens = [20 * n for n in lens]
    check_attend(a2sf, (B, 1, 1, 64, HF, 16, past, 20, lens, 0.5, "bhnd", 0.0))


def test_append_queries_in_place_and_a_cache_without_start(a2sf):
    """q_out = q; start = NULL: positions and the recent window follow from past."""
    import ctypes

    B, H, G, d, c = 2, 3, 2, 64, 5
    plan = a2sf.a2sf_rotary_plan_init(d)
    g = torch.Generator().manual_seed(12)
    q, k, v = (torch.randn((B, h, c, d), generator=g).to(HF).cuda() for h in (H * G, H, H))
    a, b = (pu.make_cache(a2sf, B, H, G, d, HF, 16, [20, 3], c, seed=6) for _ in range(2))
    b.p.start = None
    b._calls = a2sf._calls.Calls(ctypes.addressof(b.p), 0)
    want = a.a2sf_paged_append(k, v, q=q, rotary=plan)
    mine = q.clone()
    got = b.a2sf_paged_append(k, v, q=mine, q_out=mine, rotary=plan)
    assert got.data_ptr() == mine.data_ptr() and torch.equal(got, want)
    for x in (a, b):
        x.a2sf_paged_attend(want, 0.5)
        x.a2sf_paged_evict(8, 4, c)
    for name in ("k_pages", "v_pages", "scores", "positions", "past"):
        assert torch.equal(getattr(a, name).double().nan_to_num(7.0), getattr(b, name).double().nan_to_num(7.0)), name
    assert a.start.tolist() == b.start.tolist() == [20 + c, 3 + c]


def test_a_call_on_a_given_stream_allocates_there(a2sf):
    """Workspaces and outputs of a call on a given stream come from that stream's memory: work queued on the
    current stream afterwards may not get it while the call is still running."""
    B, H, d, c = 2, 8, 128, 64
    g = torch.Generator().manual_seed(13)
    q, k, v = (torch.randn((B, H, c, d), generator=g).to(BF).cuda() for _ in range(3))
    cache, ref = (pu.make_cache(a2sf, B, H, 1, d, BF, 64, [3000, 2000], c, seed=6) for _ in range(2))
    for x in (cache, ref):
        x.a2sf_paged_append(k, v)
    want = ref.a2sf_paged_attend(q, 0.9)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, lse = cache.a2sf_paged_attend(q, 0.9, stream=side)
    for _ in range(20):                                 # would land in the workspace, were it the current stream's
        torch.full((cache.attend_workspace_bytes(c) // 4,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(cache.scores.nan_to_num(7.0), ref.scores.nan_to_num(7.0))


def test_inputs_whose_rows_overlap_or_lie_apart_get_outputs_of_their_own(a2sf):
    """x[b,h,t] = row h + t of one matrix (strides of d allow it); and every third row of a larger tensor."""
    g = torch.Generator().manual_seed(14)
    H, n, d = 4, 20, 64
    base = torch.randn((H + n, d), generator=g).to(BF).cuda()
    plan = a2sf.a2sf_rotary_plan_init(d)
    for x in (base.as_strided((1, H, n, d), (0, d, d, 1)), torch.randn((1, n, 3 * H, d), generator=g).to(BF).cuda().transpose(1, 2)[:, ::3]):
        flat = x.contiguous()
        assert torch.equal(a2sf.a2sf_rotary(plan, x), a2sf.a2sf_rotary(plan, flat))
        a, b = (pu.make_cache(a2sf, 1, H, 1, d, BF, 16, [40], n, seed=6) for _ in range(2))
        assert torch.equal(a.a2sf_paged_append(flat, flat, q=x, rotary=plan), b.a2sf_paged_append(flat, flat, q=flat, rotary=plan))
        for got, want in zip(a.a2sf_paged_attend(x), b.a2sf_paged_attend(flat)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_large_values_under_logits_that_rise_by_tiles(a2sf, dtype):
    """Logits 0, 10, .. 40 in turn every 64 slots, values of 1e30: no sum before the division may overflow."""
    d, ps, L = 128, 128, 76800
    g = torch.Generator().manual_seed(15)
    cache = a2sf.PagedCache(1, 1, d, dtype, ps, L // ps, L // ps, scale=1.0)
    logit = (torch.arange(L) // 64 % 5 * 10).to(dtype)
    k, v = torch.zeros((L, d), dtype=dtype), (torch.randn((L, d), generator=g) * 1e30).to(dtype)
    k[:, 0] = logit
    cache.k_pages.copy_(k.view(-1, 1, ps, d))
    cache.v_pages.copy_(v.view(-1, 1, ps, d))
    cache.page_table.copy_(torch.arange(L // ps).view(1, -1))
    cache.past.fill_(L - 1)
    q = torch.zeros((1, 1, 1, d), dtype=dtype, device="cuda")
    q[..., 0] = 1
    out, lse = cache.a2sf_paged_attend(q, 0.5)
    o, z, s, size, _ = pu.attend_ref(k.double(), v.double(), q[0].cpu().double(), torch.zeros(L, dtype=torch.float64), L - 1, 0.5, 1.0)
    u, e = torch.finfo(dtype).eps / 2, (d + 2) * F * 40
    close(out[0], o, u * o.abs() + (u + 2 * e + 2.0 ** -20 + L * F) * size, "out")
    close(lse[0], z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), "lse")


def test_the_first_eviction_of_a_process_at_any_capacity():
    """What a kernel may take of shared memory is asked for once: the first call decides, so it is a process of its own."""
    import subprocess
    import sys
    from pathlib import Path

    code = """
import torch
from paper_2407_20485_b200 import binding as a2sf
for d, dtype in ((64, torch.bfloat16), (128, torch.bfloat16), (128, torch.float32)):
    for slots in (5120, 5632, 6016, 6144, 6272):
        cache = a2sf.PagedCache(1, 1, d, dtype, 128, slots // 128, slots // 128)
        cache.page_table.copy_(torch.arange(slots // 128).view(1, -1))
        cache.k_pages.zero_(), cache.v_pages.zero_()
        cache.scores.copy_(torch.arange(slots).view(-1, 1, 128))
        cache.positions.copy_(torch.arange(slots).view(-1, 1, 128))
        cache.past.fill_(slots - 1), cache.start.fill_(slots - 1)
        cache.a2sf_paged_evict(100, 0)
        assert cache.past.tolist() == [100] and sorted(cache.scores[0, 0, :100].tolist()) == list(range(slots - 100, slots)), slots
assert a2sf.a2sf_last_device_status() == 0
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                       cwd=Path(__file__).resolve().parent.parent)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("B,H,past,c,budget,fresh", [
    (3, 2, [90, 300, 17], 3, 250, True), (3, 2, [90, 300, 17], 3, 280, False), (5, 70, [40, 3, 0, 25, 60], 3, 30, True),
    (2, 2, [700, 100], 1, 600, True), (2, 1, [900, 850], 20, 400, False)])
def test_new_lengths_apart_from_the_old_ones(a2sf, B, H, past, c, budget, fresh):
    """past_out and start_out in arrays of their own, overlapping past by all but one entry, or past and start themselves."""
    n, ps, d = [p + c for p in past], 16, 64
    spare = -(-budget // ps)
    g = torch.Generator().manual_seed(16)
    results = []
    for how in ("same", "apart", "shifted"):
        cache = pu.make_cache(a2sf, B, H, 1, d, BF, ps, n, spare * ps, seed=4)
        cache.scores.copy_(torch.rand(cache.scores.shape, generator=torch.Generator().manual_seed(5)).mul(6).floor())
        lengths, start = torch.zeros(2 * B + 2, dtype=torch.int32), torch.tensor([p + 9 for p in past], dtype=torch.int32)
        lengths[:B] = torch.tensor(past)
        lengths, start = lengths.cuda(), start.cuda()
        pages = cache.k_pages.shape[0]
        pool = {x: torch.cat([getattr(cache, x), torch.zeros((B * spare,) + getattr(cache, x).shape[1:], device="cuda", dtype=getattr(cache, x).dtype)])
                for x in ("k_pages", "v_pages", "scores", "positions")}
        cache = a2sf.PagedCache(B, H, d, BF, ps, pages + B * spare, cache.max_pages, page_table=cache.page_table, past=lengths[:B], start=start, **pool)
        dst = (pages + torch.arange(B * spare, dtype=torch.int32)).view(B, spare).cuda() if fresh else None
        at = {"same": 0, "apart": B + 1, "shifted": 1}[how]
        past_out, start_out = lengths[at:at + B], start if how == "same" else torch.zeros_like(start)
        cache.a2sf_paged_evict(budget, 10, c, dst_table=dst, past_out=past_out, start_out=start_out)
        assert past_out.tolist() == [min(x, budget) for x in n] and start_out.tolist() == [p + 9 + c for p in past], how
        if how == "apart":
            assert lengths[:B].tolist() == past and start.tolist() == [p + 9 for p in past]
        results.append([getattr(cache, x).double().nan_to_num(7.0) for x in pool])
    assert all(torch.equal(x, y) for r in results[1:] for x, y in zip(results[0], r))


@pytest.mark.parametrize("kind", ["last bits", "equal scores", "equal pairs", "wide positions"])
@pytest.mark.parametrize("heads,n,drop", [(1, 500, 100), (200, 300, 60)])
def test_evict_where_most_bits_are_shared(a2sf, kind, heads, n, drop):
    """Scores that differ in their last bits only, scores or (score, position) pairs that are all equal, positions of all sizes."""
    ps = 16
    cache = pu.make_cache(a2sf, 1, heads, 1, 64, BF, ps, [n], 0, seed=3)
    g = torch.Generator().manual_seed(18)
    table, j = cache.page_table.cpu()[0].long(), torch.arange(n)
    bits = torch.full((heads, n), 0x3f800000, dtype=torch.int32)
    if kind == "last bits":
        bits += torch.randint(0, 200, (heads, n), generator=g).to(torch.int32)
    score = bits.view(torch.float32)
    pos = torch.full((heads, n), 77, dtype=torch.int32)
    if kind == "wide positions":
        pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (heads, n), generator=g).to(torch.int32)
    elif kind != "equal pairs":
        pos = torch.stack([torch.randperm(n, generator=g) for _ in range(heads)]).to(torch.int32)
    cpu = {x: getattr(cache, x).cpu() for x in ("scores", "positions", "k_pages")}
    cpu["scores"][table[j // ps], :, j % ps] = score.T
    cpu["positions"][table[j // ps], :, j % ps] = pos.T
    cache.scores.copy_(cpu["scores"])
    cache.positions.copy_(cpu["positions"])
    cache.past.fill_(n - 1)
    cache.start.fill_(2 ** 31 - 2)                              # nothing is recent
    M = n - drop
    cache.a2sf_paged_evict(M, 0)
    got = {x: getattr(cache, x).cpu()[table[j[:M] // ps], :, j[:M] % ps] for x in cpu}
    for h in range(heads):
        order = sorted(range(n), key=lambda s: (float(score[h, s]), int(pos[h, s]), s))
        stay = set(order[drop:])
        holes, ups = [s for s in range(M) if s not in stay], [s for s in range(M, n) if s in stay]
        src = list(range(M))
        for hole, up in zip(holes, ups):
            src[hole] = up
        src = torch.tensor(src)
        for x in cpu:
            assert torch.equal(got[x][:, h], cpu[x][table[src // ps], h, src % ps]), (kind, h, x)


@pytest.mark.parametrize("case", [
    (20, 3, 1, 64, FP, 16, [600 - 7 * b for b in range(20)], 200, [200 - 9 * b for b in range(20)], 0.9, "bhnd", 0.0),
    (20, 2, 3, 128, FP, 64, [3 * b for b in range(20)], 173, None, 1.0, "bnhd", 0.0),
    (1, 2, 1, 128, FP, 32, [5000], 33, [31], 0.5, "bhnd", 0.0),
    (2, 1, 4, 64, FP, 128, [2999, 0], 50, [50, 17], 0.99, "bnhd", 0.0)], ids=["many-pieces", "many", "few-long", "few-group"])
def test_attend_in_32_bits_in_large_tiles_and_in_pieces(a2sf, case):
    check_attend(a2sf, case, seed=21)


# ---- many rows in 16-bit storage on tcgen05: calls that are large by the capacity of their page tables ------------

def room_for_large(case):
    """Slots behind `past` that make the call large: 3e8 multiply-adds of Q K^T at capacity, 1.2e9 for up to 64 rows."""
    B, H, G, d, _, _, _, c = case[:8]
    return int((1.3e9 if c * G <= 64 else 3.3e8) / (B * H * G * c * d))


LARGE = [c for c in ATT if c[4] != FP and c[2] * c[7] > 16] + [
    (6, 4, 1, 128, BF, 64, [500, 0, 63, 64, 65, 1300], 40, [40, 40, 0, 1, 39, 40], 0.9, "bhnd", 0.0),
    (2, 2, 4, 128, HF, 32, [0, 600], 200, [200, 150], 1.0, "bnhd", 0.0),           # a capacity of 800 slots: no plan
    (3, 4, 2, 64, BF, 16, [0, 300, 128], 290, [290, 0, 129], 0.5, "bhnd", 0.0)]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "") for x in c))
def test_attend_of_large_calls(a2sf, case):
    if case[7] * case[2] == 17:
        case = (3, 5) + case[2:6] + ([0, 70, 129],) + case[7:]
    check_attend(a2sf, case, room=room_for_large(case), seed=31)


@pytest.mark.parametrize("seed", range(24))
def test_attend_random_large_calls(a2sf, seed):
    r = random.Random(1000 + seed)
    while True:
        case = random_attend(r)
        if case[4] != FP and case[2] * case[7] > 64:
            break
    check_attend(a2sf, case, seed=seed + 300, room=room_for_large(case))


@pytest.mark.parametrize("dtype,G,c,past,gain,garbage", [
    (BF, 2, 150, 200, 12.0, math.nan), (HF, 2, 150, 200, 12.0, math.nan), (BF, 4, 40, 33, 1.0, math.inf), (HF, 2, 150, 0, 1.0, math.inf)])
def test_large_logits_and_infinities_in_large_calls(a2sf, dtype, G, c, past, gain, garbage):
    case = (2, 2, G, 128, dtype, 32, [past, 1], c, [c, c - 3], 0.9, "bhnd", 0.0)
    check_attend(a2sf, case, seed=9, gain=gain, garbage=garbage, room=room_for_large(case))


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, "pages", "past", "length"])
def test_bad_pages_and_lengths_in_large_calls(a2sf, bad):
    c = 150
    cache = pu.make_cache(a2sf, 2, 2, 1, 128, HF, 16, [40, 30], 8000, seed=4, garbage=0.0)
    lens = torch.full((2,), c, dtype=torch.int32, device="cuda")
    if bad == "past":
        cache.past[1] = cache.max_pages * 16 + 5
    elif bad == "length":
        lens[1] = -4
    else:
        cache.page_table[1, :] = cache.num_pages if bad == "pages" else bad
    x = torch.randn((2, 2, c, 128), device="cuda").to(HF)
    cache.a2sf_paged_attend(x, 0.5, lens=lens)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_ERR_INVALID_ARG
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK


def test_a_large_call_captured_and_replayed(a2sf):
    B, H, G, d, c = 2, 2, 2, 128, 200
    g = torch.Generator().manual_seed(33)
    ins = [[torch.randn((B, h, c, d), generator=g).to(BF).cuda() for h in (H * G, H, H)] for _ in range(3)]
    a, b = (pu.make_cache(a2sf, B, H, G, d, BF, 32, [300, 5], 8000, seed=6) for _ in range(2))
    q, k, v = (x.clone() for x in ins[0])
    out, lse = torch.empty_like(q), torch.empty((B, H * G, c), device="cuda")

    def step(cache, q, k, v, out, lse):
        cache.a2sf_paged_append(k, v)
        cache.a2sf_paged_attend(q, 0.9, out=out, lse=lse)
        cache.a2sf_paged_evict(1000, 8, c)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, q, k, v, out, lse)
    for x in ins:
        for dst, src in zip((q, k, v), x):
            dst.copy_(src)
        graph.replay()
        o2, z2 = torch.empty_like(q), torch.empty_like(lse)
        step(b, *x, o2, z2)
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(lse, z2)
        for name in ("k_pages", "scores", "positions", "past", "start"):
            assert torch.equal(getattr(a, name).double().nan_to_num(7.0), getattr(b, name).double().nan_to_num(7.0)), name


def test_a_large_call_far_inside_a_large_pool(a2sf):
    """Pages beyond 2^31 elements, read through a table of 40 entries, give what the same pages give in a small pool."""
    H, d, ps, past, c = 8, 128, 128, 300, 130
    pages = (2 ** 31) // (H * ps * d) + 40
    far = torch.zeros((1, 40), dtype=torch.int32)
    near = far.clone()
    far[0, :4], near[0, :4] = pages - 1 - torch.arange(4), torch.tensor([2, 0, 3, 1])
    g = torch.Generator().manual_seed(5)
    k, v, q = (torch.randn((1, H, past + c, d), generator=g).to(HF).cuda() for _ in range(3))
    results = []
    for n_pages, table in ((pages, far), (4, near)):
        cache = a2sf.PagedCache(1, H, d, HF, ps, n_pages, 40, page_table=table.cuda())
        cache.a2sf_paged_append(k, v)
        cache.past.fill_(past)
        out, lse = cache.a2sf_paged_attend(q[:, :, past:], 0.9)
        results.append((out.cpu(), lse.cpu(), pu.slots(cache, cache.scores.cpu(), 0, past + c)))
        del cache
    for x, y in zip(*results):
        assert torch.equal(x, y)
