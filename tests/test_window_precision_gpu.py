"""How exact every form of the windowed attention is, on inputs where a rounding of the probabilities would show.

Keys are made for given logits (log2 units): q = (1, 2^-9, 0, ..), k = (hi, lo, 0, ..), scale = ln 2; the reference takes what
is stored.  u = torch.finfo(dtype).eps / 2 is the half step of the storage type, F = 2^-24 that of fp32."""
import math

import pytest
import torch

from window_forms import FORMS, attend, expected

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
LN2 = float(torch.tensor(math.log(2), dtype=FP))
HALVES = [name for name in FORMS if FORMS[name][4] != FP]
BELOW = {"cluster": 13, "whole": 13, "list": 13, "mma": 15, "tcgen05": 8}       # of the reference under the maximum, fp16, log2 units


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import binding

    return binding


def visible(past, c, window, sinks):
    p, j = past + torch.arange(c)[:, None], torch.arange(past + c)[None, :]
    return (j <= p) & ((j < sinks) | (j > p - window))


def run(a2sf, name, dtype, k, values, scale=math.log(2), ps=64):
    """Windowed attention in the named form over sequences and heads that all hold keys k [L][d] and values [L], by queries (1, 2^-9, 0, ..)
    -> out [B, H*G, c, d], lse, and of one head in 64 bits: out [c], lse [c], sum P|V| [c]."""
    B, H, G, d, _, past, c, window, sinks = FORMS[name]
    L = past + c
    pages = -(-L // ps)
    cache = a2sf.PagedCache(B, H, d, dtype, ps, pages, pages, group=G, scale=scale)
    for pool, x in ((cache.k_pages, k.to(dtype)), (cache.v_pages, values.to(dtype)[:, None].expand(L, d))):
        rows = torch.zeros((pages * ps, d), dtype=dtype)
        rows[:L] = x
        pool.copy_(rows.view(pages, 1, ps, d).expand(pages, H, ps, d))
    cache.page_table.copy_(torch.arange(pages, dtype=torch.int32).expand(B, pages))       # read only: sequences share their pages
    cache.past.fill_(past)
    q = torch.zeros((B, H * G, c, d), dtype=dtype, device="cuda")
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -9
    out, lse, form = attend(a2sf, cache, q, window, sinks)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK
    assert form == expected(name)
    kd, v = k.to(dtype).double(), values.to(dtype).double()
    x = ((kd[:, 0] + kd[:, 1] / 512) * float(torch.tensor(scale, dtype=FP)))[None, :].masked_fill(~visible(past, c, window, sinks), -math.inf)
    z = torch.logsumexp(x, -1)
    P = torch.exp(x - z[:, None])
    return out.cpu().double(), lse.cpu().double(), P @ v, z, P @ v.abs()


def keys(logits, d, dtype):
    k = torch.zeros((logits.numel(), d), dtype=torch.float64)
    k[:, 0] = logits.to(dtype).double()
    k[:, 1] = (logits - k[:, 0]) * 512
    return k


def compare(out, o, tol, what):
    worst = float(((out - o).abs() / tol).nan_to_num(math.inf).max())
    assert worst <= 1, f"{what}: {worst:.3g} of the tolerance"


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("name", HALVES)
def test_terms_of_a_probability(a2sf, name, dtype):
    """Half of the keys have a probability just below the middle of two neighbours of the storage type, half just above, and values 1
    and -1: what is left of their sum is a tenth of what rounding to one term adds, 0.9 u of it.  Two terms are off by u^2, and all forms but
    tcgen05 keep two."""
    B, H, G, d, _, past, c, window, sinks = FORMS[name]
    L, u = past + c, torch.finfo(dtype).eps / 2
    j = torch.arange(L)
    kind = torch.where(j % 8 == 0, torch.zeros_like(j), 1 + j % 2)              # every eighth key: logit 0 and value 0
    p = torch.tensor([1.0, 0.5 + 0.45 * u, 0.5 + 0.55 * u], dtype=torch.float64)[kind]      # u between neighbours from 1/2 on
    values = torch.tensor([0.0, 1.0, -1.0], dtype=torch.float64)[kind]
    out, lse, o, z, size = run(a2sf, name, dtype, keys(torch.log2(p), d, dtype), values)
    most = int(visible(past, c, window, sinks).sum(1).max())
    e = (d + 2) * F * 2                                                        # logits of -1 and 0, from products of 1 at most
    under = 0.0 if dtype != HF else 2.0 ** -25 * most                          # fp16 below its normal range
    terms = u if name.startswith("tcgen05") else u * u
    tol = u * o.abs() + (terms + 2 * e + 2.0 ** -20 + most * F) * size + under
    seen = visible(past, c, window, sinks).double()
    one = seen @ (p.to(dtype).double() * values) / (seen @ p)                  # with one term: these values would show it
    assert bool(((one - o).abs() > tol).all()) == (not name.startswith("tcgen05"))
    compare(out, o[:, None], tol[:, None], name)
    compare(lse, z, e + 2.0 ** -20 + most * F + 4 * F * z.abs(), f"lse, {name}")


@pytest.mark.parametrize("sink", ["every", "first"])
@pytest.mark.parametrize("name", HALVES)
def test_small_probabilities_in_fp16(a2sf, name, sink):
    """Keys of equal, small probability beside one (or every sixteenth) that draws nearly everything and has value 0: the output is
    the others' share.  fp16 holds a probability to half a step down to 2^-14 and to 2^-25 absolutely below, against a reference
    2^BELOW under the maximum."""
    B, H, G, d, _, past, c, window, sinks = FORMS[name]
    L, u = past + c, 2.0 ** -11
    j = torch.arange(L)
    at = j % 16 == 0 if sink == "every" else j == 0
    seen = visible(past, c, window, sinks)
    n, heavy = seen.sum(1).double(), (seen & at).sum(1).double()
    weight = torch.where(heavy > 0, heavy, n)                                  # of the row, in units of its largest
    values = torch.where(at, 0.0, 1000.0).double()
    terms = u if name.startswith("tcgen05") else u * u
    least = 2.0 ** -25 / 2.0 ** BELOW[name.split(",")[0]]
    for small in (25.01, 24.45, 22.3, 17.6, 13.7, 30.0):
        out, lse, o, z, size = run(a2sf, name, HF, keys(torch.where(at, 0.0, -small).double(), d, HF), values)
        e = 6 * F * small                                                      # two products that are not zero, the sum, the scale
        under = least * n * 1000 / weight
        compare(out, o[:, None], (u * o.abs() + 2.0 ** -25 + (terms + 2 * e + 2.0 ** -20 + n * F) * size + under)[:, None], f"{name}, 2^-{small}")
        compare(lse, z, e + 2.0 ** -20 + n * F + 4 * F * z.abs(), f"lse, {name}, 2^-{small}")


@pytest.mark.parametrize("name,dtype", [(name, BF if name in HALVES else FP) for name in FORMS])
def test_values_up_to_the_stated_bound(a2sf, name, dtype):
    """Values of nearly 2^113 / slots, all of one sign, under logits that rise and fall by tiles within what a reference may be
    exceeded by: no sum before the division overflows."""
    B, H, G, d, _, past, c, window, sinks = FORMS[name]
    L, u = past + c, torch.finfo(dtype).eps / 2
    j = torch.arange(L)
    logits = (j // 64 % 4 * 4.5 + (j % 64 == 9) * 0.25).double()
    values = torch.full((L,), 0.99 * 2.0 ** 113 / L, dtype=torch.float64)
    out, lse, o, z, size = run(a2sf, name, dtype, keys(logits, d, dtype), values)
    most, e = int(visible(past, c, window, sinks).sum(1).max()), 6 * F * 14
    compare(out, o[:, None], (u * o.abs() + (u + 2 * e + 2.0 ** -20 + most * F) * size)[:, None], name)
    compare(lse, z, e + 2.0 ** -20 + 4 * F * z.abs() + most * F, f"lse, {name}")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("place", [2, 8, 16])
@pytest.mark.parametrize("name", HALVES)
def test_logits_whose_last_place_is_a_power_of_the_probability(a2sf, name, place, dtype):
    """Logits of 1.5e7 last places that rise and fall by up to 30 of them: a last place of 2 (log2 units) or more rounds what is
    subtracted before the exponential.  With values of 1 the output is 1 whatever the probabilities; none may leave the type's
    range."""
    B, H, G, d, _, past, c, window, sinks = FORMS[name]
    L, u = past + c, torch.finfo(dtype).eps / 2
    j = torch.arange(L)
    k = torch.zeros((L, d), dtype=torch.float64)
    k[:, 0], k[:, 1] = 59904.0, (j // 64 % 4 * 20 + j % 16).div(2).floor().mul(2).double()
    scale = 256 * place * math.log(2)
    out, lse, _, _, _ = run(a2sf, name, dtype, k, torch.ones(L, dtype=torch.float64), scale=scale)
    most = int(visible(past, c, window, sinks).sum(1).max())
    terms = u if name.startswith("tcgen05") else u * u
    compare(out, torch.ones(()), torch.tensor(u + terms + 2.0 ** -20 + most * F), name)
    # the largest logit is one that the row sees; the sum adds ln of the slots at most
    x = ((59904 + k[:, 1] / 512) * float(torch.tensor(scale, dtype=FP)))[None, :].masked_fill(~visible(past, c, window, sinks), -math.inf)
    top = x.max(1).values
    assert float((lse - top).abs().max()) <= math.log(most) + 4 * place * math.log(2), f"lse, {name}"
