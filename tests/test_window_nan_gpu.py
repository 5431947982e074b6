"""A NaN among the keys of a windowed attention shows in every row that sees it, and in no other, whatever form the call takes: also
where all that one warp or one piece of a cut row saw is NaN, so that its partial result has no finite part."""
import math

import pytest
import torch

from test_window_gpu import F, HF, close, window_ref
from window_forms import FORMS, attend, expected

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import binding

    return binding


def filled(a2sf, B, H, G, d, dtype, past, c, ps=32, seed=4):
    """Sequences of past + c tokens, the same keys and values in all of them -> cache (past set), K, V [H][L][d], q."""
    g = torch.Generator().manual_seed(seed)
    L = past + c
    pages = -(-L // ps)
    k, v = (torch.randn((H, pages * ps, d), generator=g).to(dtype) for _ in range(2))
    cache = a2sf.PagedCache(B, H, d, dtype, ps, pages, pages, group=G)
    for pool, x in ((cache.k_pages, k), (cache.v_pages, v)):
        pool.copy_(x.view(H, pages, ps, d).transpose(0, 1))
    cache.page_table.copy_(torch.arange(pages, dtype=torch.int32).expand(B, pages))       # read only: sequences share their pages
    cache.past.fill_(past)
    q = torch.randn((B, H * G, c, d), generator=g).to(dtype).cuda()
    return cache, k[:, :L], v[:, :L], q


# a slot, all that a warp takes of a tile, and more than a piece of a row has (eight tiles of 128 slots)
@pytest.mark.parametrize("run", [1, 32, 1024])
@pytest.mark.parametrize("name", FORMS)
def test_a_nan_key_shows_in_every_row_that_sees_it(a2sf, name, run):
    B, H, G, d, dtype, past, c, window, sinks = FORMS[name]
    cache, K, V, q = filled(a2sf, B, H, G, d, dtype, past, c)
    L, ps = past + c, cache.page_size
    p, j = past + torch.arange(c)[:, None], torch.arange(L)[None, :]
    seen = (j <= p) & ((j < sinks) | (j > p - window))
    # aligned in the window of the last row, where that goes; ending with the last slot; a first slot that later rows no longer see
    lo = max(0, L - window)
    places = {max(lo, (lo + 2 * (L - lo) // 3 - run) // 32 * 32), L - min(run, L - lo), max(lo - c // 2, 0)}
    for at in places:
        bad = torch.zeros(L, dtype=torch.bool)
        bad[at : at + run] = True
        for h in (0, H - 1):
            whole = cache.k_pages.clone()
            flat = cache.k_pages[:, h].reshape(-1, d)
            flat[at : at + run] = math.nan
            cache.k_pages[:, h] = flat.view(-1, ps, d)
            out, lse, form = attend(a2sf, cache, q, window, sinks)
            assert form == expected(name)
            hit = (seen & bad).any(1)
            assert hit.any()
            for b in (0, B - 1):
                rows = slice(h * G, (h + 1) * G)
                o, z, size, logit, most, vmax = window_ref(K[h].double().masked_fill(bad[:, None], 0.0), V[h].double(), q[b, rows].cpu().double(), past, window, sinks,
                                                           1 / math.sqrt(d))
                u, e = torch.finfo(dtype).eps / 2, (d + 2) * F * logit
                under = 0.0 if dtype != HF else 2.0 ** -25 * most * vmax
                tol = u * o.abs() + (u + 2 * e + 2.0 ** -20 + most * F) * size + under
                assert bool(out[b, rows][:, hit.cuda()].isnan().all()) and bool(lse[b, rows][:, hit.cuda()].isnan().all()), f"{at}, head {h}: a NaN went missing"
                close(out[b, rows][:, (~hit).cuda()], o[:, ~hit], tol[:, ~hit], f"out {at} {b} {h}")
                close(lse[b, rows][:, (~hit).cuda()], z[:, ~hit], (e + 2.0 ** -20 + 4 * F * z.abs())[:, ~hit], f"lse {at} {b} {h}")
                if H > 1:                                  # other heads see none of it
                    other = [x for x in range(H) if x != h]
                    assert not bool(out[b].view(H, G, c, d)[other].isnan().any())
            cache.k_pages.copy_(whole)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK
