"""Refusals of the rotary and paged-cache entry points, and the rotary plan's arithmetic: host only, no GPU."""
import ctypes
import math

import pytest
import torch

import paged_util as pu


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import build

    build.build()
    from paper_2407_20485_b200 import binding

    return binding


INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -5
OK, ODD = 0x10000, 0x10008


def _paged(a2sf, **kw):
    p = a2sf.a2sf_paged(2, 3, 2, 128, 1, 64, 40, 8, 0.0, 0, *([OK] * 7))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


S = (6 * 5 * 128, 5 * 128, 128)      # strides of a [2][6][5][128] tensor
SKV = (3 * 5 * 128, 5 * 128, 128)


def _append(a2sf, p, plan=None, c=5, k=OK, v=OK, skv=SKV, q=None, q_out=None, sq=S, so=S, lens=None):
    return a2sf.lib.a2sf_paged_append(ctypes.byref(p) if p is not None else None, None if plan is None else ctypes.byref(plan), c, lens,
                                      k, v, *skv, q, *sq, q_out, *so, None)


def _attend(a2sf, p, c=5, alpha=0.5, q=OK, sq=S, out=OK + 4096, so=S, lse=None, flags=0, ws=OK, nbytes=1 << 40, lens=None):
    return a2sf.lib.a2sf_paged_attend(ctypes.byref(p) if p is not None else None, c, lens, alpha, q, *sq, out, *so, lse, flags, ws, nbytes, None)


def _evict(a2sf, p, c=5, budget=100, recent=10, dst=None, dst_pages=0, past=OK, start=OK + 64, ws=OK, nbytes=1 << 40):
    return a2sf.lib.a2sf_paged_evict(ctypes.byref(p) if p is not None else None, c, None, budget, recent, dst, dst_pages, past, start, ws, nbytes, None)


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, INVALID), ("B", 1025, UNSUPPORTED), ("H", 0, INVALID), ("group", 0, UNSUPPORTED), ("group", 9, UNSUPPORTED),
    ("d", 96, UNSUPPORTED), ("dtype", 3, UNSUPPORTED), ("page_size", 48, UNSUPPORTED), ("page_size", 8, UNSUPPORTED),
    ("num_pages", 0, INVALID), ("max_pages", 0, INVALID), ("max_pages", 1 << 23, UNSUPPORTED), ("num_pages", 1 << 30, UNSUPPORTED),
    ("scale", -1.0, INVALID), ("scale", float("nan"), INVALID), ("scale", float("inf"), INVALID), ("reserved", 1, INVALID),
    ("k_pages", None, INVALID), ("v_pages", ODD, INVALID), ("scores", None, INVALID), ("positions", None, INVALID),
    ("page_table", None, INVALID), ("past", None, INVALID), ("past", OK + 2, INVALID), ("start", OK + 1, INVALID),
])
def test_a_bad_cache_is_refused_by_every_call(a2sf, field, value, status):
    p = _paged(a2sf, **{field: value})
    assert _append(a2sf, p) == status
    assert _attend(a2sf, p) == status
    assert _evict(a2sf, p) == status
    assert a2sf.lib.a2sf_paged_attend_workspace_bytes(ctypes.byref(p), 5) == 0
    assert a2sf.lib.a2sf_paged_evict_workspace_bytes(ctypes.byref(p), 100) == 0


def test_bad_arguments_of_the_calls(a2sf):
    p, plan = _paged(a2sf), a2sf.a2sf_rotary_plan_init(128)
    assert _append(a2sf, None) == INVALID and _attend(a2sf, None) == INVALID and _evict(a2sf, None) == INVALID
    for bad in (dict(c=0), dict(k=None), dict(v=ODD), dict(skv=(SKV[0], SKV[1], 100)), dict(skv=(SKV[0], SKV[1] + 4, 128)),
                dict(skv=(0, SKV[1], 128)), dict(lens=OK + 2), dict(q=OK, q_out=OK),                      # q without a plan
                dict(plan=plan, q=OK), dict(plan=plan, q=ODD, q_out=OK), dict(plan=plan, q=OK, q_out=OK, so=(S[0] * 2, S[1], S[2])),
                dict(plan=a2sf.a2sf_rotary_plan())):
        assert _append(a2sf, p, **bad) == INVALID, bad
    assert _append(a2sf, _paged(a2sf, d=64), plan=plan) == INVALID                                        # rotary_dim > d
    for bad in (dict(c=0), dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=float("nan")), dict(q=None), dict(out=None), dict(q=ODD),
                dict(out=OK), dict(sq=(S[0], S[1], 64)), dict(so=(S[0], 1, 128)), dict(flags=2), dict(lse=OK + 2), dict(ws=None), dict(ws=OK + 128)):
        assert _attend(a2sf, p, **bad) == INVALID, bad
    assert _attend(a2sf, p, nbytes=16) == WORKSPACE
    for bad in (dict(budget=0), dict(recent=-1), dict(recent=101), dict(past=None), dict(start=None), dict(past=OK, start=OK),
                dict(dst=OK, dst_pages=0), dict(dst=OK, dst_pages=1), dict(dst=OK + 2, dst_pages=8), dict(ws=None), dict(ws=OK + 16)):
        assert _evict(a2sf, p, **bad) == INVALID, bad
    assert _evict(a2sf, p, nbytes=16) == WORKSPACE
    # axes of extent 1 may have any stride
    one = _paged(a2sf, B=1, H=1, group=1)
    assert _attend(a2sf, one, c=1, sq=(0, 3, 7), so=(0, 0, 0), nbytes=16) == WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=130), dict(rotary_dim=64, theta=1.0), dict(rotary_dim=64, theta=float("inf")),
    dict(rotary_dim=64, factor=0.5), dict(rotary_dim=2, scaling="ntk", factor=2.0), dict(rotary_dim=64, scaling="bands", factor=2.0),
    dict(rotary_dim=64, scaling="ramp", factor=2.0, original_length=4096, low=4.0, high=4.0), dict(rotary_dim=64, magnitude=-1.0),
    dict(rotary_dim=64, scaling="bands", factor=2.0, original_length=4096, low=0.0),
])
def test_bad_rotary_configurations(a2sf, kw):
    with pytest.raises(a2sf.A2SFError) as e:
        a2sf.a2sf_rotary_plan_init(**kw)
    assert e.value.status == INVALID
    with pytest.raises(ValueError):
        a2sf.a2sf_rotary_plan_init(64, scaling="cubic")


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 3.0), ("bands", 8.0), ("ramp", 16.0)])
@pytest.mark.parametrize("r", [4, 24, 64, 126, 128])
def test_the_plan_holds_the_frequencies(a2sf, r, scaling, factor):
    """turn[k] / 2^64 of a turn is f_k / 2 pi to the double's accuracy (1e-15 relatively, and 2^-64 absolutely)."""
    high = 32.0 if scaling == "ramp" else 4.0
    plan = a2sf.a2sf_rotary_plan_init(r, theta=500000.0, scaling=scaling, factor=factor, original_length=8192, low=1.0, high=high)
    want = pu.inv_freq(r, 500000.0, scaling, factor, 8192, 1.0, high)
    for k, f in enumerate(want):
        got = plan.turn[k] / 2.0 ** 64 * 2 * math.pi
        assert abs(got - f) <= 4e-15 * f + 2.0 ** -61
    assert all(plan.turn[k] == 0 for k in range(len(want), 64))
    assert plan.magnitude == pytest.approx(0.1 * math.log(factor) + 1 if scaling == "ramp" else 1.0, rel=1e-6)
    assert a2sf.a2sf_rotary_plan_init(r, magnitude=1.5).magnitude == 1.5


def test_bad_rotary_calls(a2sf):
    plan = a2sf.a2sf_rotary_plan_init(64)

    def call(plan=plan, dtype=1, B=2, H=3, n=5, d=64, x=OK, xs=(960, 320, 64), y=OK, ys=(960, 320, 64), positions=None, start=None, lens=None, flags=0):
        return a2sf.lib.a2sf_rotary(None if plan is None else ctypes.byref(plan), dtype, B, H, n, d, x, *xs, y, *ys, positions, start, lens, flags, None)

    assert call(dtype=5) == UNSUPPORTED and call(d=80) == UNSUPPORTED
    for bad in (dict(plan=None), dict(plan=a2sf.a2sf_rotary_plan()), dict(B=0), dict(H=0), dict(n=0), dict(x=None), dict(y=ODD),
                dict(xs=(960, 320, 60)), dict(xs=(960, 0, 64)), dict(ys=(1920, 320, 64)), dict(flags=2), dict(start=OK + 1),
                dict(positions=OK + 2), dict(lens=OK + 3)):
        assert call(**bad) == INVALID, bad
    assert call(plan=a2sf.a2sf_rotary_plan_init(128)) == INVALID


def test_the_binding_refuses_tensors_of_other_shapes_types_and_places(a2sf):
    cache = a2sf.PagedCache(2, 3, 64, torch.bfloat16, 16, 10, 4, group=2, device="cpu")
    q, k = torch.zeros((2, 6, 5, 64), dtype=torch.bfloat16), torch.zeros((2, 3, 5, 64), dtype=torch.bfloat16)
    for call in (lambda: cache.a2sf_paged_attend(q[:, :3]), lambda: cache.a2sf_paged_attend(q.half()),
                 lambda: cache.a2sf_paged_attend(q.transpose(2, 3).contiguous().transpose(2, 3)),
                 lambda: cache.a2sf_paged_attend(q, lse=torch.zeros((2, 6, 4))),
                 lambda: cache.a2sf_paged_attend(q, lens=torch.zeros(3, dtype=torch.int32)),
                 lambda: cache.a2sf_paged_attend(q, lens=torch.zeros(2, dtype=torch.int64)),
                 lambda: cache.a2sf_paged_append(k, k[:, :2]), lambda: cache.a2sf_paged_append(k, k.transpose(1, 2).contiguous().transpose(1, 2)),
                 lambda: cache.a2sf_paged_evict(5, 1, dst_table=torch.zeros((3, 2), dtype=torch.int32)),
                 lambda: a2sf.PagedCache(2, 3, 64, torch.bfloat16, 16, 10, 4, k_pages=torch.zeros(1))):
        with pytest.raises(ValueError):
            call()


def test_the_binding_refuses_numbers_of_more_than_32_bits(a2sf):
    cache = a2sf.PagedCache(2, 3, 64, torch.bfloat16, 16, 10, 4, device="cpu")
    for bad in (dict(budget=2 ** 32 + 5, recent=1), dict(budget=5, recent=2 ** 32 + 1), dict(budget=5, recent=1, c=2 ** 32 + 1)):
        with pytest.raises(ValueError, match="32-bit"):
            cache.a2sf_paged_evict(**bad)
