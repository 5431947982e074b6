"""How exact the attention over the paged cache is, on inputs where a rounding of the probabilities would show.

Keys are made for given logits (log2 units): q = (1, 2^-9, 0, ..), k = (hi, lo, 0, ..), scale = ln 2; the reference takes what
is stored.  u = torch.finfo(dtype).eps / 2 is the half step of the storage type, F = 2^-24 that of fp32."""
import math

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


def run(a2sf, B, H, G, d, dtype, c, logits, values, room=0, ps=64):
    """Attention of the last c tokens of sequences that all hold these logits and values [L] -> out, lse of every head and
    the 64-bit out, lse, sum P|V| of one."""
    L = logits.numel()
    hi = logits.to(dtype)
    k, v = torch.zeros((L, d), dtype=dtype), values.to(dtype)[:, None].expand(L, d).contiguous()
    k[:, 0], k[:, 1] = hi, ((logits - hi.double()) * 512).to(dtype)
    pages = -(-L // ps)
    cache = a2sf.PagedCache(B, H, d, dtype, ps, B * pages, max(pages, -(-(L + room) // ps)), group=G, scale=math.log(2))
    pad = torch.zeros((pages * ps, d), dtype=dtype)
    for pool, x in ((cache.k_pages, k), (cache.v_pages, v)):
        pad[:L] = x
        pool.copy_(pad.view(1, pages, 1, ps, d).expand(B, pages, H, ps, d).reshape(B * pages, H, ps, d))
    cache.page_table[:, :pages] = torch.arange(B * pages, dtype=torch.int32).view(B, pages)
    cache.past.fill_(L - c)
    q = torch.zeros((B, H * G, c, d), dtype=dtype, device="cuda")
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -9
    out, lse = cache.a2sf_paged_attend(q, 0.9)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK
    want = pu.attend_ref(k.double(), v.double(), q[0, :1].cpu().double(), torch.zeros(L, dtype=torch.float64), L - c, 0.9,
                         float(torch.tensor(math.log(2), dtype=FP)))
    return out.cpu().double(), lse.cpu().double(), want[0], want[1], want[3]


def compare(out, o, tol, what):
    worst = float(((out - o).abs() / tol).max())
    assert worst <= 1, f"{what}: {worst:.3g} of the tolerance"


PATHS = {
    # B, H, G, d, c, L
    "whole units": (1, 2, 1, 128, 1, 200), "whole units, 64": (2, 2, 2, 64, 2, 300), "whole units, 8 rows": (1, 2, 8, 128, 1, 150),
    "split": (2, 2, 1, 128, 1, 4000), "split, 64": (1, 3, 3, 64, 1, 5000), "split, 8 rows": (2, 1, 4, 128, 2, 3000),
    "split, 16 rows": (2, 2, 4, 64, 4, 3000), "small tiles": (1, 3, 1, 128, 40, 333), "small tiles, pieces": (1, 1, 2, 64, 30, 3000),
    "large tiles": (60, 10, 1, 64, 64, 128)}


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("path", PATHS)
def test_probabilities_keep_two_terms_of_the_storage_type(a2sf, path, dtype):
    """Half of the keys have a probability just below the middle of two neighbours of the storage type, half just above, and
    values 1 and -1: what is left of their sum is a tenth of what rounding to one term would add.  Two terms are off by u^2."""
    B, H, G, d, c, L = PATHS[path]
    u = torch.finfo(dtype).eps / 2
    j = torch.arange(L)
    kind = torch.where(j % 8 == 0, torch.zeros_like(j), 1 + j % 2)              # every eighth key: logit 0 and value 0
    step = u                                                                   # between neighbours from 1/2 on
    p = torch.tensor([1.0, 0.5 + 0.45 * step, 0.5 + 0.55 * step], dtype=torch.float64)[kind]
    values = torch.tensor([0.0, 1.0, -1.0], dtype=torch.float64)[kind]
    out, lse, o, z, size = run(a2sf, B, H, G, d, dtype, c, torch.log2(p), values)
    e = (d + 2) * F * 2                                                        # logits of -1 and 0, from products of 1 at most
    under = 0.0 if dtype != HF else 2.0 ** -25 * L                             # fp16 below its normal range
    compare(out, o, u * o.abs() + (u * u + 2 * e + 2.0 ** -20 + L * F) * size + under, path)
    compare(lse, z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs(), path)


# tcgen05: large by the capacity of the page table (`room` slots behind the sequence), with a plan and pieces; direct; two row tiles of a group
LARGE = {"tcgen05": (1, 2, 1, 128, 130, 3000, 8000), "tcgen05, direct": (8, 8, 1, 128, 200, 700, 0), "tcgen05, group": (2, 1, 3, 64, 100, 2000, 20000)}
BELOW = {"whole": 13, "split": 13, "small": 15, "large": 15, "tcgen05": 8}       # of the reference under the maximum, log2 units


@pytest.mark.parametrize("sink", ["every", "first", "last"])
@pytest.mark.parametrize("path", [*PATHS, *LARGE])
def test_small_probabilities_in_fp16(a2sf, path, sink):
    """Keys of equal, small probability beside one (or every sixteenth) that draws nearly everything and has value 0: the output is
    the others' share.  fp16 holds a probability to half a step down to 2^-14 and to 2^-25 absolutely below, against a reference
    2^BELOW under the maximum."""
    B, H, G, d, c, L, room = (PATHS.get(path) or LARGE[path])[:6] + (LARGE.get(path, (0,) * 7)[6],)
    u = 2.0 ** -11
    j = torch.arange(L)
    at = j % 16 == 0 if sink == "every" else j == (0 if sink == "first" else L - c)
    values = torch.where(at, 0.0, 1000.0).double()
    terms = u if path in LARGE else u * u
    least = 2.0 ** -25 / 2.0 ** BELOW[path.split(",")[0].split(" ")[0]]
    for small in (25.01, 24.45, 22.3, 17.6, 13.7, 30.0):
        out, lse, o, z, size = run(a2sf, B, H, G, d, HF, c, torch.where(at, 0.0, -small).double(), values, room)
        e = 6 * F * small                                                      # two products that are not zero, the sum, the scale
        seen = L - c + 1 + torch.arange(c, dtype=torch.float64)[None, :, None]
        weight = torch.floor((seen + 15) / 16) if sink == "every" else 1.0     # of the row, in units of the largest
        under = least * seen * 1000 / weight
        compare(out, o, u * o.abs() + 2.0 ** -25 + (terms + 2 * e + 2.0 ** -20 + L * F) * size + under, f"{path}, 2^-{small}")
        compare(lse, z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs() + L * F, path)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("path", [*PATHS, *LARGE])
def test_values_up_to_the_stated_bound(a2sf, path, dtype):
    """Values of nearly 2^113 / slots, all of one sign, under logits that rise and fall by tiles within what a reference may be
    exceeded by: no sum before the division overflows."""
    B, H, G, d, c, L, room = (PATHS.get(path) or LARGE[path])[:6] + (LARGE.get(path, (0,) * 7)[6],)
    u = torch.finfo(dtype).eps / 2
    j = torch.arange(L)
    logits = (j // 64 % 4 * 4.5 + (j % 64 == 9) * 0.25).double()
    values = torch.full((L,), 0.99 * 2.0 ** 113 / L, dtype=torch.float64)
    out, lse, o, z, size = run(a2sf, B, H, G, d, dtype, c, logits, values, room)
    e = 6 * F * 14
    compare(out, o, u * o.abs() + (u + 2 * e + 2.0 ** -20 + L * F) * size, path)
    compare(lse, z, torch.full_like(z, e + 2.0 ** -20) + 4 * F * z.abs() + L * F, path)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("place", [2, 8, 16])
@pytest.mark.parametrize("path", [*PATHS, *LARGE])
def test_logits_whose_last_place_is_a_power_of_the_probability(a2sf, path, place, dtype):
    """Logits of 1.5e7 last places that rise and fall by up to 30 of them: a last place of 2 (log2 units) or more rounds what is
    subtracted before the exponential.  With values of 1 the output is 1 whatever the probabilities; none may leave the type's
    range."""
    B, H, G, d, c, L, room = (PATHS.get(path) or LARGE[path])[:6] + (LARGE.get(path, (0,) * 7)[6],)
    u, ps = torch.finfo(dtype).eps / 2, 64
    pages = -(-L // ps)
    j = torch.arange(pages * ps)
    k = torch.zeros((pages * ps, d), dtype=dtype)
    k[:, 0], k[:, 1] = 59904.0, (j // 64 % 4 * 20 + j % 16).div(2).floor().mul(2).to(dtype)
    cache = a2sf.PagedCache(B, H, d, dtype, ps, B * pages, max(pages, -(-(L + room) // ps)), group=G, scale=256 * place * math.log(2))
    cache.k_pages.copy_(k.view(1, pages, 1, ps, d).expand(B, pages, H, ps, d).reshape(B * pages, H, ps, d))
    cache.v_pages.fill_(1.0)
    cache.page_table[:, :pages] = torch.arange(B * pages, dtype=torch.int32).view(B, pages)
    cache.past.fill_(L - c)
    q = torch.zeros((B, H * G, c, d), dtype=dtype, device="cuda")
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -9
    out, lse = cache.a2sf_paged_attend(q, 0.9)
    assert a2sf.a2sf_last_device_status() == a2sf.A2SF_OK
    terms = u if path in LARGE else u * u
    compare(out.cpu().double(), torch.ones(()), torch.tensor(u + terms + 2.0 ** -20 + L * F), path)
    # the largest logit is one that the row sees; the sum adds ln L at most
    seen = (59904 + k[:L, 1].double() / 512).cummax(0).values[L - c:] * float(torch.tensor(256 * place * math.log(2), dtype=FP))
    worst = float((lse.cpu().double() - seen).abs().max())
    assert worst <= math.log(L) + 4 * place * math.log(2), worst
