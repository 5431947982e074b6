"""Refusals of the calls for rotary positions with several axes and for windowed attention, and the axes' plan: host only, no GPU."""
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
S, SKV = (6 * 5 * 128, 5 * 128, 128), (3 * 5 * 128, 5 * 128, 128)      # strides of [2][6][5][128] and [2][3][5][128]


def _paged(a2sf, **kw):
    p = a2sf.a2sf_paged(2, 3, 2, 128, 1, 64, 40, 8, 0.0, 0, *(OK + 4096 * x for x in range(7)))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _append(a2sf, p, plan, positions=OK, c=5, k=OK, v=OK, skv=SKV, q=None, q_out=None, sq=S, so=S, lens=None):
    return a2sf.lib.a2sf_paged_append_axes(_ref(p), _ref(plan), positions, c, lens, k, v, *skv, q, *sq, q_out, *so, None)


def _window(a2sf, p, c=5, window=7, sinks=2, q=OK, sq=S, out=OK + 4096, so=S, lse=None, ws=OK, nbytes=1 << 40, lens=None):
    return a2sf.lib.a2sf_paged_attend_window(_ref(p), c, lens, window, sinks, q, *sq, out, *so, lse, ws, nbytes, None)


FAR = 0x900000


def _slide(a2sf, p, c=5, window=7, sinks=2, table=FAR, freed=FAR + 4096, count=FAR + 8192, past=FAR + 12288, start=FAR + 16384, lens=None):
    return a2sf.lib.a2sf_paged_slide(_ref(p), c, lens, window, sinks, table, freed, count, past, start, None)


def _plan(a2sf, pairs=(16, 24, 24), **kw):
    return a2sf.a2sf_rotary_axes_plan_init(pairs, a2sf.a2sf_rotary_plan_init(2 * sum(pairs), **kw))


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, INVALID), ("B", 1025, UNSUPPORTED), ("H", 0, INVALID), ("group", 9, UNSUPPORTED), ("d", 96, UNSUPPORTED), ("dtype", 3, UNSUPPORTED),
    ("page_size", 48, UNSUPPORTED), ("num_pages", 0, INVALID), ("max_pages", 1 << 23, UNSUPPORTED), ("scale", float("nan"), INVALID),
    ("reserved", 1, INVALID), ("k_pages", None, INVALID), ("v_pages", ODD, INVALID), ("page_table", None, INVALID), ("past", OK + 2, INVALID),
])
def test_a_bad_cache_is_refused_by_every_call(a2sf, field, value, status):
    p = _paged(a2sf, **{field: value})
    assert _append(a2sf, p, _plan(a2sf)) == status
    assert _window(a2sf, p) == status
    assert _slide(a2sf, p) == status
    assert a2sf.lib.a2sf_paged_attend_window_workspace_bytes(ctypes.byref(p), 5, 7, 2) == 0


def test_bad_arguments_of_append_with_axes(a2sf):
    p, plan = _paged(a2sf), _plan(a2sf)
    assert _append(a2sf, None, plan) == INVALID and _append(a2sf, p, None) == INVALID
    for bad in (dict(c=0), dict(positions=None), dict(positions=OK + 2), dict(k=None), dict(v=ODD), dict(skv=(SKV[0], SKV[1], 100)),
                dict(skv=(0, SKV[1], 128)), dict(lens=OK + 2), dict(q=OK), dict(q=ODD, q_out=OK), dict(q=OK, q_out=OK, so=(S[0] * 2, S[1], S[2]))):
        assert _append(a2sf, p, plan, **bad) == INVALID, bad
    assert _append(a2sf, _paged(a2sf, d=64), plan) == INVALID                            # rotary_dim > d
    # a plan of another kind, one that was never made, and one whose axes were overwritten
    assert a2sf.lib.a2sf_paged_append_axes(ctypes.byref(p), ctypes.byref(a2sf.a2sf_rotary_plan_init(128)), OK, 5, None, OK, OK, *SKV, None, *S, None, *S, None) == INVALID
    assert _append(a2sf, p, a2sf.a2sf_rotary_axes_plan()) == INVALID
    plan.axis[63] = 3
    assert _append(a2sf, p, plan) == INVALID
    assert a2sf.lib.a2sf_paged_append(ctypes.byref(p), ctypes.byref(_plan(a2sf)), 5, None, OK, OK, *SKV, None, *S, None, *S, None) == INVALID


def test_bad_arguments_of_windowed_attention(a2sf):
    p = _paged(a2sf)
    assert _window(a2sf, None) == INVALID
    for bad in (dict(c=0), dict(window=0), dict(window=-1), dict(sinks=-1), dict(q=None), dict(out=None), dict(q=ODD), dict(out=OK),
                dict(sq=(S[0], S[1], 64)), dict(so=(S[0], 1, 128)), dict(lse=OK + 2), dict(ws=None), dict(ws=OK + 128), dict(lens=OK + 1)):
        assert _window(a2sf, p, **bad) == INVALID, bad
    assert _window(a2sf, p, nbytes=16) == WORKSPACE
    need = lambda c, w, s: a2sf.lib.a2sf_paged_attend_window_workspace_bytes(ctypes.byref(p), c, w, s)  # noqa: E731
    assert need(0, 7, 2) == need(5, 0, 2) == need(5, 7, -1) == 0
    for c in (1, 5, 200):
        assert need(c, 1, 0) > 0 and need(c, 2 ** 31 - 1, 2 ** 31 - 1) == need(c, 512, 512)        # beyond the capacity nothing grows
        assert _window(a2sf, p, c=c, sq=(6 * c * 128, c * 128, 128), so=(6 * c * 128, c * 128, 128), nbytes=need(c, 7, 2) - 1) == WORKSPACE


def test_the_workspace_follows_the_window_and_not_the_capacity(a2sf):
    small, large = (a2sf.a2sf_paged(4, 8, 4, 128, 1, 64, 1 << 16, mp, 0.0, 0, *([OK] * 7)) for mp in (64, 4096))
    for c in (1, 4, 100, 2000):
        a, b = (a2sf.lib.a2sf_paged_attend_window_workspace_bytes(ctypes.byref(p), c, 1024, 4) for p in (small, large))
        assert a == b > 0


def test_bad_arguments_of_slide(a2sf):
    p = _paged(a2sf)
    assert _slide(a2sf, None) == INVALID
    table, past, start = p.page_table, p.past, p.start
    for bad in (dict(c=0), dict(window=0), dict(sinks=-1), dict(table=None), dict(past=None), dict(start=None), dict(table=FAR + 2), dict(freed=FAR + 1),
                dict(count=FAR + 3), dict(past=FAR + 2), dict(lens=OK + 2), dict(freed=table), dict(freed=FAR), dict(freed=FAR + 4), dict(count=past),
                dict(count=start), dict(past=start), dict(start=past), dict(past=past + 4), dict(start=start - 4), dict(table=table + 4),
                dict(past=FAR, start=FAR), dict(lens=FAR + 12288), dict(lens=FAR + 12292), dict(count=FAR + 12284)):
        assert _slide(a2sf, p, **bad) == INVALID, bad


@pytest.mark.parametrize("pairs,plans,cycle", [
    ([], [64], False), ([0, 32], [64], False), ([33, 32], [130], False), ([8] * 5, [80], False), ([16, 16], [62], False),
    ([16, 16], [32, 34], False), ([16, 8, 8], [32, 16], False), ([16, -1], [64], True), ([65], [64], False),
])
def test_bad_plans_of_several_axes(a2sf, pairs, plans, cycle):
    with pytest.raises((a2sf.A2SFError, ValueError)):
        a2sf.a2sf_rotary_axes_plan_init(pairs, [a2sf.a2sf_rotary_plan_init(r) for r in plans], cycle=cycle)


def test_plans_of_the_axes_must_agree_and_be_plans(a2sf):
    make, raw = a2sf.a2sf_rotary_plan_init, a2sf.lib.a2sf_rotary_axes_plan_init
    for other in (make(32, interleaved=True), make(32, magnitude=1.5), a2sf.a2sf_rotary_plan()):
        with pytest.raises(a2sf.A2SFError):
            a2sf.a2sf_rotary_axes_plan_init([16, 16], [make(32), other])
    with pytest.raises(ValueError):
        a2sf.a2sf_rotary_axes_plan_init([16, 16], [None])
    pairs, out, plan = (ctypes.c_int32 * 2)(16, 16), a2sf.a2sf_rotary_axes_plan(), make(64)
    assert raw(2, pairs, 0, ctypes.byref(plan), 1, ctypes.byref(out)) == 0
    for args in ((0, pairs, 0, ctypes.byref(plan), 1, ctypes.byref(out)), (2, None, 0, ctypes.byref(plan), 1, ctypes.byref(out)),
                 (2, pairs, 2, ctypes.byref(plan), 1, ctypes.byref(out)), (2, pairs, 0, None, 1, ctypes.byref(out)),
                 (2, pairs, 0, ctypes.byref(plan), 3, ctypes.byref(out)), (2, pairs, 0, ctypes.byref(plan), 1, None)):
        assert raw(*args) == INVALID


@pytest.mark.parametrize("pairs", [[1], [64], [16, 24, 24], [24, 20, 20], [2, 5], [1, 1, 1, 61], [7, 3, 2, 9]])
@pytest.mark.parametrize("cycle", [False, True])
@pytest.mark.parametrize("each", [False, True])
def test_the_plan_gives_every_pair_its_axis_and_frequency(a2sf, pairs, cycle, each):
    rest, axis = list(pairs), []
    while sum(rest):                                   # dealt by hand
        for a in range(len(rest)):
            take = 0 if not rest[a] else 1 if cycle else rest[a]
            axis += [a] * take
            rest[a] -= take
    make = lambda r: a2sf.a2sf_rotary_plan_init(r, theta=300.0, interleaved=True, scaling="linear", factor=3.0)  # noqa: E731
    plan = a2sf.a2sf_rotary_axes_plan_init(pairs, [make(2 * n) for n in pairs] if each else make(2 * sum(pairs)), cycle=cycle)
    assert plan.rotary_dim == 2 * sum(pairs) and plan.interleaved == 1 and plan.magnitude == 1.0 and plan.axes == len(pairs)
    assert [plan.axis[k] for k in range(64)] == axis + [0] * (64 - len(axis))
    seen = [0] * len(pairs)
    for k, a in enumerate(axis):
        f = 300.0 ** (-seen[a] / pairs[a]) / 3.0 if each else 300.0 ** (-k / sum(pairs)) / 3.0
        seen[a] += 1
        assert abs(plan.turn[k] / 2.0 ** 64 * 2 * math.pi - f) <= 4e-15 * f + 2.0 ** -61
    assert all(plan.turn[k] == 0 for k in range(len(axis), 64))
    assert pu.inv_freq(8)[0] == 1.0


def test_a_copied_plan_is_a_plan_of_its_own(a2sf):
    import copy

    plan = _plan(a2sf)
    other = copy.copy(plan)
    assert other.at == ctypes.addressof(other) != plan.at and bytes(other) == bytes(plan)
    assert _append(a2sf, _paged(a2sf, d=64), other) == INVALID           # read as a plan: rotary_dim > d


def test_bad_rotations_with_several_axes(a2sf):
    plan = _plan(a2sf, (8, 12, 12))

    def call(plan=plan, dtype=1, B=2, H=3, n=5, d=64, x=OK, xs=(960, 320, 64), y=OK, ys=(960, 320, 64), positions=OK, lens=None, flags=0):
        return a2sf.lib.a2sf_rotary_axes(_ref(plan), dtype, B, H, n, d, x, *xs, y, *ys, positions, lens, flags, None)

    assert call(dtype=5) == UNSUPPORTED and call(d=80) == UNSUPPORTED
    for bad in (dict(plan=None), dict(plan=a2sf.a2sf_rotary_axes_plan()), dict(B=0), dict(H=0), dict(n=0), dict(x=None), dict(y=ODD), dict(xs=(960, 320, 60)),
                dict(xs=(960, 0, 64)), dict(ys=(1920, 320, 64)), dict(flags=2), dict(positions=None), dict(positions=OK + 2), dict(lens=OK + 3),
                dict(plan=_plan(a2sf))):
        assert call(**bad) == INVALID, bad


def test_the_binding_refuses_tensors_of_other_shapes_types_and_places(a2sf):
    cache = a2sf.PagedCache(2, 3, 64, torch.bfloat16, 16, 10, 4, group=2, device="cpu")
    q, k = torch.zeros((2, 6, 5, 64), dtype=torch.bfloat16), torch.zeros((2, 3, 5, 64), dtype=torch.bfloat16)
    plan, pos, i32 = _plan(a2sf, (8, 12, 12)), torch.zeros((3, 2, 5), dtype=torch.int32), torch.int32
    for call in (lambda: cache.a2sf_paged_attend_window(q[:, :3], 4), lambda: cache.a2sf_paged_attend_window(q.half(), 4),
                 lambda: cache.a2sf_paged_attend_window(q.transpose(2, 3).contiguous().transpose(2, 3), 4),
                 lambda: cache.a2sf_paged_attend_window(q, 4, lse=torch.zeros((2, 6, 4))), lambda: cache.a2sf_paged_attend_window(q, 4, lens=torch.zeros(3, dtype=i32)),
                 lambda: cache.a2sf_paged_attend_window(q, 2 ** 32 + 4), lambda: cache.a2sf_paged_attend_window(q, 4, 2 ** 32),
                 lambda: cache.a2sf_paged_append_axes(k, k, pos[:2], plan), lambda: cache.a2sf_paged_append_axes(k, k, pos.long(), plan),
                 lambda: cache.a2sf_paged_append_axes(k, k[:, :2], pos, plan), lambda: cache.a2sf_paged_append_axes(k, k, pos, a2sf.a2sf_rotary_plan_init(64)),
                 lambda: cache.a2sf_paged_append_axes(k, k, pos, None),
                 lambda: cache.a2sf_paged_append_axes(k, k, pos.transpose(1, 2).contiguous().transpose(1, 2), plan),
                 lambda: cache.a2sf_paged_slide(4, table_out=torch.zeros((2, 3), dtype=i32)), lambda: cache.a2sf_paged_slide(4, freed=torch.zeros((2, 4))),
                 lambda: cache.a2sf_paged_slide(4, c=2 ** 32 + 1), lambda: cache.a2sf_paged_slide(4, freed_count=torch.zeros(3, dtype=i32)),
                 lambda: cache.a2sf_paged_slide(4),                                          # all in order, but not on a GPU
                 lambda: a2sf.a2sf_rotary_axes(plan, k[0], pos), lambda: a2sf.a2sf_rotary_axes(plan, k, pos[:, :1]),
                 lambda: a2sf.a2sf_rotary_axes(a2sf.a2sf_rotary_plan_init(64), k, pos), lambda: a2sf.a2sf_rotary_axes(plan, k, pos)):
        with pytest.raises(ValueError):
            call()
