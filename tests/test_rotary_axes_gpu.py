"""Rotary positions with several axes, alone and on the way into the paged cache, against plain 64-bit forms on a B200.

Tolerances as for one axis: an angle is off by less than 3e-8, sine and cosine by that and 2e-7 with what sincospi leaves, the two
products and the sum by 4 f of the pair's length (f = 2^-24); then the rounding to the storage type."""
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
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - want).abs() / tol.clamp_min(1e-300)).max()):.3g} of the tolerance"


def axes_of(pairs, cycle):
    """(axis, index in the axis) of every pair, dealt by hand."""
    rest, done, out = list(pairs), [0] * len(pairs), []
    while sum(rest):
        for a in range(len(rest)):
            for _ in range(0 if not rest[a] else 1 if cycle else rest[a]):
                out.append((a, done[a]))
                done[a] += 1
                rest[a] -= 1
    return out


def turn(x, pos, pairs, cycle, each, theta, interleaved, transpose=False):
    """x [h][n][d] in 64 bits, pos [axes][n]: pair by pair."""
    y, h = x.clone(), sum(pairs)
    for k, (a, j) in enumerate(axes_of(pairs, cycle)):
        f = theta ** (-j / pairs[a]) if each else theta ** (-k / h)
        p, q = (2 * k, 2 * k + 1) if interleaved else (k, k + h)
        ang = pos[a].double() * f
        c, s = torch.cos(ang), torch.sin(ang) * (-1 if transpose else 1)
        y[..., p] = x[..., p] * c - x[..., q] * s
        y[..., q] = x[..., q] * c + x[..., p] * s
    return y


def make_plan(a2sf, pairs, cycle, each, theta, interleaved):
    make = lambda r: a2sf.a2sf_rotary_plan_init(r, theta=theta, interleaved=interleaved)  # noqa: E731
    return a2sf.a2sf_rotary_axes_plan_init(pairs, [make(2 * n) for n in pairs] if each else make(2 * sum(pairs)), cycle=cycle)


def places(g, A, B, n, far):
    """Positions of every kind: small grids, far ones of either sign, the same on all axes for the first tokens."""
    p = torch.randint(-far, far, (A, B, n), generator=g)
    p[:, :, : n // 3] = torch.arange(n // 3)
    return p.to(torch.int32)


ROT = [
    # B, H, n, d, dtype, pairs, cycle, each, interleaved, transpose, far, layout
    (1, 1, 1, 64, BF, [16, 8, 8], False, False, False, False, 10, "bhnd"),
    (2, 5, 37, 128, BF, [16, 24, 24], False, False, False, False, 5000, "bnhd"),
    (2, 5, 37, 128, HF, [24, 20, 20], True, False, False, True, 100000, "bhnd"),
    (3, 2, 33, 64, FP, [9, 7], True, True, True, True, 2 ** 31 - 1, "bhnd"),
    (1, 3, 65, 64, FP, [1, 2, 3, 6], True, False, False, False, 2 ** 31 - 1, "bnhd"),
    (2, 4, 19, 128, HF, [11, 1], False, True, False, True, 900, "bhnd"),
    (2, 3, 5, 64, BF, [1, 1], True, True, True, False, 77, "bhnd"),
    (1, 40, 130, 128, BF, [22, 21, 21], True, True, True, False, 50000, "bnhd"),
    (4, 1, 257, 128, FP, [63], False, False, False, False, 12345, "bhnd"),
    (2, 7, 300, 128, HF, [61, 1, 1, 1], True, False, True, False, 70000, "bhnd"),
]


@pytest.mark.parametrize("case", ROT, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "") for x in c))
def test_rotary_axes(a2sf, case):
    B, H, n, d, dtype, pairs, cycle, each, il, transpose, far, layout = case
    g = torch.Generator().manual_seed(1)
    plan = make_plan(a2sf, pairs, cycle, each, 10000.0, il)
    x = torch.randn((B, H, n, d) if layout == "bhnd" else (B, n, H, d), generator=g).to(dtype)
    xc = x.cuda() if layout == "bhnd" else x.cuda().transpose(1, 2)
    x = x if layout == "bhnd" else x.transpose(1, 2)
    pos = places(g, len(pairs), B, n, far)
    lens = torch.tensor([n if b == 0 else max(0, n - 4 * b) for b in range(B)], dtype=torch.int32)
    want = torch.stack([turn(x[b].double(), pos[:, b].long(), pairs, cycle, each, 10000.0, il, transpose) for b in range(B)])
    out = torch.full_like(xc, 9.0)
    got = a2sf.a2sf_rotary_axes(plan, xc, pos.cuda(), out=out, lens=lens.cuda(), transpose=transpose)
    live = (torch.arange(n) < lens[:, None])[:, None, :, None]
    # the reference's own angle in 64 bits is off by 2^-53 of it
    tol = torch.finfo(dtype).eps / 2 * want.abs() + x.double().norm(dim=-1, keepdim=True) * (2e-7 + 4 * F + far * 2.0 ** -52)
    close(torch.where(live.cuda(), got, torch.zeros_like(got)), torch.where(live, want, torch.zeros_like(want)), tol, "rotary")
    assert bool((got == 9.0)[~live.cuda().expand_as(got)].all()), "rows past the length were written"
    r = 2 * sum(pairs)
    assert bool((got.cpu()[..., r:] == x[..., r:])[live.expand_as(x)[..., r:]].all()), "elements past rotary_dim are copies"
    again = a2sf.a2sf_rotary_axes(plan, xc, pos.cuda(), out=xc, lens=lens.cuda(), transpose=transpose)        # in place
    assert again.data_ptr() == xc.data_ptr() and torch.equal(again[live.cuda().expand_as(again)], got[live.cuda().expand_as(got)])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pairs,cycle", [([32], False), ([10, 12, 10], True)])
def test_equal_positions_on_all_axes_are_the_rotation_of_one(a2sf, dtype, pairs, cycle):
    g = torch.Generator().manual_seed(2)
    x = torch.randn((3, 4, 50, 64), generator=g).to(dtype).cuda()
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, 50), generator=g).to(torch.int32).cuda()
    base = a2sf.a2sf_rotary_plan_init(64, scaling="ramp", factor=4.0, original_length=4096, low=1.0, high=32.0)
    plan = a2sf.a2sf_rotary_axes_plan_init(pairs, base, cycle=cycle)
    got = a2sf.a2sf_rotary_axes(plan, x, pos.expand(len(pairs), -1, -1).contiguous())
    assert torch.equal(got, a2sf.a2sf_rotary(base, x, positions=pos))


def test_gradient_by_differences_and_inverse(a2sf):
    plan = make_plan(a2sf, [8, 12, 12], True, False, 500.0, False)
    g = torch.Generator().manual_seed(3)
    x, dy, e = (torch.randn((2, 3, 9, 64), generator=g).cuda() for _ in range(3))
    pos = places(g, 3, 2, 9, 1000).cuda()
    dx = a2sf.a2sf_rotary_axes(plan, dy, pos, transpose=True)
    h = 0.5              # y is linear in x: <dy, y(x + h e) - y(x)> / h = <dx, e>, up to the rounding of the two forward passes
    diff = ((a2sf.a2sf_rotary_axes(plan, x + h * e, pos).double() - a2sf.a2sf_rotary_axes(plan, x, pos).double()) * dy.double()).sum() / h
    tol = 8 * (2e-7 + 4 * F) * float((x.norm() + e.norm()) * dy.norm() / h)
    assert abs(float(diff - (dx.double() * e.double()).sum())) <= tol
    back = a2sf.a2sf_rotary_axes(plan, a2sf.a2sf_rotary_axes(plan, x, pos), pos, transpose=True)
    assert float((back - x).abs().max()) <= 2 * (2e-7 + 4 * F) * float(x.norm(dim=-1).max())


def check_append(a2sf, B, H, G, d, dtype, ps, c, pairs, cycle, each, il, layout, seed=4):
    past = [(5 * b + 3) % 41 for b in range(B)]
    cache = pu.make_cache(a2sf, B, H, G, d, dtype, ps, past, c, seed=2)
    before = {x: getattr(cache, x).cpu().clone() for x in ("k_pages", "v_pages", "scores", "positions")}
    start = torch.tensor([1000 * b + 7 for b in range(B)], dtype=torch.int32)
    cache.start.copy_(start)
    g = torch.Generator().manual_seed(seed)
    lens = torch.tensor([c if b == 0 else (c * (b + 1)) % (c + 1) for b in range(B)], dtype=torch.int32)

    def tensor(h):
        t = torch.randn((B, h, c, d), generator=g).to(dtype)
        return t, (t.cuda() if layout == "bhnd" else t.transpose(1, 2).contiguous().cuda().transpose(1, 2))

    (k, kc), (v, vc), (q, qc) = tensor(H), tensor(H), tensor(H * G)
    pos, plan = places(g, len(pairs), B, c, 30000), make_plan(a2sf, pairs, cycle, each, 10000.0, il)
    q_out = torch.full_like(qc, 5.0)
    got = cache.a2sf_paged_append_axes(kc, vc, pos.cuda(), plan, lens=lens.cuda(), q=qc, q_out=q_out)
    assert got.data_ptr() == q_out.data_ptr()
    want = {x: t.clone().double() if t.is_floating_point() else t.clone() for x, t in before.items()}
    tol, table, u = torch.zeros_like(want["k_pages"]), cache.page_table.cpu(), torch.finfo(dtype).eps / 2
    for b in range(B):
        kr, qr = (turn(x[b].double(), pos[:, b].long(), pairs, cycle, each, 10000.0, il) for x in (k, q))
        n = int(lens[b])
        for t in range(n):
            pg, o = int(table[b, (past[b] + t) // ps]), (past[b] + t) % ps
            want["k_pages"][pg, :, o], want["v_pages"][pg, :, o] = kr[:, t], v[b, :, t].double()
            tol[pg, :, o] = u * kr[:, t].abs() + k[b, :, t].double().norm(dim=-1, keepdim=True) * (2e-7 + 4 * F)
            want["scores"][pg, :, o], want["positions"][pg, :, o] = 0, int(start[b]) + t
        close(got[b, :, :n], qr[:, :n], u * qr[:, :n].abs() + q[b, :, :n].double().norm(dim=-1, keepdim=True) * (2e-7 + 4 * F), "q")
        assert bool((got[b, :, n:] == 5.0).all())
    garbage = torch.isnan(want["k_pages"])
    assert torch.equal(torch.isnan(cache.k_pages.cpu()), garbage), "slots outside the chunk were touched"
    close(torch.where(garbage.cuda(), torch.zeros_like(cache.k_pages), cache.k_pages), want["k_pages"].nan_to_num(0.0), tol, "keys")
    for x in ("v_pages", "scores"):
        assert torch.equal(getattr(cache, x).cpu().double().nan_to_num(7.0), want[x].nan_to_num(7.0)), x
    assert torch.equal(cache.positions.cpu(), want["positions"]) and cache.past.tolist() == past


@pytest.mark.parametrize("B,H,G,d,dtype,ps,c,pairs,cycle,each,il,layout", [
    (1, 1, 1, 64, FP, 16, 1, [16, 8, 8], False, False, False, "bhnd"),
    (3, 2, 4, 128, BF, 32, 37, [16, 24, 24], False, False, False, "bnhd"),
    (2, 5, 3, 128, HF, 64, 130, [7, 5], True, True, True, "bhnd"),
    (4, 3, 8, 64, HF, 128, 5, [4, 3, 3], True, False, False, "bnhd"),
])
def test_append_axes(a2sf, B, H, G, d, dtype, ps, c, pairs, cycle, each, il, layout):
    check_append(a2sf, B, H, G, d, dtype, ps, c, pairs, cycle, each, il, layout)


@pytest.mark.parametrize("seed", range(16))
def test_append_axes_random_cases(a2sf, seed):
    r = random.Random(seed)
    d, A = r.choice([64, 128]), r.choice([1, 2, 3, 4])
    most = r.choice([d // 2, d // 2, 12, 7])
    cuts = sorted(r.sample(range(1, most), A - 1))
    pairs = [y - x for x, y in zip([0] + cuts, cuts + [most])]
    check_append(a2sf, r.choice([1, 2, 5]), r.choice([1, 2, 3, 9]), r.choice([1, 2, 3, 8]), d, r.choice([FP, BF, HF]), r.choice([16, 32, 64, 128]),
                 r.choice([1, 2, 17, 100]), pairs, r.random() < 0.5, r.random() < 0.5, r.random() < 0.5, r.choice(["bhnd", "bnhd"]), seed=seed + 50)


def test_positions_of_tokens_behind_the_length_are_not_read_for_the_result(a2sf):
    """Whatever stands there, the rows before the length get the same bits, keys alone or with queries."""
    plan = make_plan(a2sf, [8, 12, 12], False, False, 10000.0, False)
    g = torch.Generator().manual_seed(6)
    k, v, q = (torch.randn((2, h, 9, 64), generator=g).to(BF).cuda() for h in (2, 2, 4))
    lens, pos = torch.tensor([5, 0], dtype=torch.int32).cuda(), places(g, 3, 2, 9, 99).cuda()
    other = pos.clone()
    other[:, 0, 5:] = 2 ** 31 - 1
    other[:, 1] = -2 ** 31
    pools = []
    for p, with_q in ((pos, True), (other, True), (other, False)):
        cache = pu.make_cache(a2sf, 2, 2, 2, 64, BF, 16, [20, 3], 9, seed=6)
        cache.a2sf_paged_append_axes(k, v, p, plan, lens=lens, q=q if with_q else None)
        pools.append(cache.k_pages.nan_to_num(7.0))
    assert torch.equal(pools[0], pools[1]) and torch.equal(pools[0], pools[2])
