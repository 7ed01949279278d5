"""Refusals of the paged cache's entry points, through the C ABI and the binding.  Nothing is launched: no GPU needed."""

import ctypes
import os

import pytest
import torch

import paper_2602_07721_amd as pk
import workloads

pytestmark = pytest.mark.skipif(not os.path.exists(pk.LIB_PATH), reason="library not built")

FAKE = 0x10000
f16, f32, i32, u8 = torch.float16, torch.float32, torch.int32, torch.uint8


def _cfg(hkv=2, g=4):
    return pk.Config(hkv, g, 1, workloads.rotation_signs(3))


def _vp(x):
    return ctypes.c_void_p(x)


def _pages(K=FAKE, V=FAKE, n=10, size=16):
    return ctypes.byref(pk._Pages(K, V, n, size))


def _step(**change):
    a = dict(table=FAKE, table_width=8, free_pages=FAKE, n_pages=10, page_size=16, n_free=FAKE, lens=FAKE, counts=FAKE, batch=2,
             t=5, new_lens=FAKE, new_free=FAKE, offsets=FAKE, granted=FAKE, slots=FAKE, positions=FAKE)
    a.update(change)
    return pk.lib().pariskv_plan_pages(ctypes.byref(pk._PageStep(**a)), None)


@pytest.mark.parametrize("name", ["table", "free_pages", "n_free", "lens", "counts", "new_lens", "new_free", "offsets", "granted",
                                  "slots", "positions"])
def test_plan_refuses_arrays(name):
    assert _step(**{name: 0}) == pk.ERR_INVALID
    assert _step(**{name: FAKE + 2}) == pk.ERR_INVALID


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), pk.ERR_INVALID), (dict(batch=65536), pk.ERR_UNSUPPORTED), (dict(table_width=0), pk.ERR_INVALID),
    (dict(table_width=2 ** 30), pk.ERR_INVALID), (dict(n_pages=0), pk.ERR_INVALID), (dict(page_size=0), pk.ERR_INVALID),
    (dict(page_size=-16), pk.ERR_INVALID), (dict(n_pages=2 ** 26), pk.ERR_INVALID), (dict(t=-1), pk.ERR_INVALID),
    (dict(t=2 ** 24 + 1), pk.ERR_UNSUPPORTED)])
def test_plan_refuses_sizes(change, code):
    assert _step(**change) == code
    assert pk.lib().pariskv_plan_pages(None, None) == pk.ERR_INVALID


@pytest.mark.parametrize("change,code", [
    (dict(q=0), pk.ERR_INVALID), (dict(k=FAKE + 8), pk.ERR_INVALID), (dict(v=0), pk.ERR_INVALID), (dict(out=FAKE + 2), pk.ERR_INVALID),
    (dict(positions=0), pk.ERR_INVALID), (dict(slots=FAKE + 1), pk.ERR_INVALID), (dict(freqs=0), pk.ERR_INVALID),
    (dict(freqs=FAKE + 2), pk.ERR_INVALID), (dict(qw=FAKE + 2), pk.ERR_INVALID), (dict(kw=FAKE + 1), pk.ERR_INVALID),
    (dict(rot=8), pk.ERR_INVALID), (dict(rot=144), pk.ERR_INVALID), (dict(rot=-16), pk.ERR_INVALID), (dict(pairs=2), pk.ERR_INVALID),
    (dict(eps=-1.0), pk.ERR_INVALID), (dict(eps=float("nan")), pk.ERR_INVALID), (dict(qs=1016), pk.ERR_INVALID),
    (dict(qs=1028), pk.ERR_INVALID), (dict(ks=128), pk.ERR_INVALID), (dict(vs=2 ** 33), pk.ERR_INVALID), (dict(t=-1), pk.ERR_INVALID),
    (dict(t=2 ** 24 + 1), pk.ERR_UNSUPPORTED), (dict(pages=None), pk.ERR_INVALID), (dict(pages=_pages(K=0)), pk.ERR_INVALID),
    (dict(pages=_pages(V=FAKE + 8)), pk.ERR_INVALID), (dict(pages=_pages(n=0)), pk.ERR_INVALID),
    (dict(pages=_pages(size=0)), pk.ERR_INVALID), (dict(pages=_pages(n=2 ** 30)), pk.ERR_INVALID)])
def test_rotate_rows_refuses(change, code):
    a = dict(pages=_pages(), q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, t=4, positions=FAKE, slots=FAKE, freqs=FAKE, rot=128,
             pairs=0, qw=0, kw=0, eps=1e-6, out=FAKE)
    a.update(change)
    assert pk.lib().pariskv_rotate_rows(
        _cfg().c(), a["pages"], _vp(a["q"]), a["qs"], _vp(a["k"]), a["ks"], _vp(a["v"]), a["vs"], a["t"], _vp(a["positions"]),
        _vp(a["slots"]), _vp(a["freqs"]), a["rot"], a["pairs"], _vp(a["qw"]), _vp(a["kw"]), ctypes.c_float(a["eps"]), _vp(a["out"]),
        None) == code


def test_pools_past_31_bits_of_rows_are_refused():
    many = pk.Config(1024, 1, 1, workloads.rotation_signs(3))
    L = pk.lib()
    args = [_vp(FAKE), 131072, _vp(FAKE), 131072, _vp(FAKE), 131072, 0, None, None, None, 0, 0, None, None, ctypes.c_float(0), None, None]
    assert L.pariskv_rotate_rows(many.c(), _pages(n=131072, size=16), *args) == pk.ERR_UNSUPPORTED
    assert L.pariskv_rotate_rows(many.c(), _pages(n=131071, size=16), *args) == pk.OK


@pytest.mark.parametrize("change,code", [
    (dict(q=0), pk.ERR_INVALID), (dict(q=FAKE + 8), pk.ERR_INVALID), (dict(out=0), pk.ERR_INVALID), (dict(table=0), pk.ERR_INVALID),
    (dict(lens=FAKE + 2), pk.ERR_INVALID), (dict(offsets=0), pk.ERR_INVALID), (dict(counts=FAKE + 2), pk.ERR_INVALID),
    (dict(slopes=FAKE + 1), pk.ERR_INVALID), (dict(width=0), pk.ERR_INVALID), (dict(width=2 ** 30), pk.ERR_INVALID),
    (dict(qs=1000), pk.ERR_INVALID), (dict(scale=float("inf")), pk.ERR_INVALID), (dict(cap=-1.0), pk.ERR_INVALID),
    (dict(cap=float("nan")), pk.ERR_INVALID), (dict(cap=1e-7), pk.ERR_INVALID), (dict(cap=1e31), pk.ERR_INVALID),
    (dict(cap=float("inf")), pk.ERR_INVALID), (dict(most=0), pk.ERR_INVALID), (dict(t=-1), pk.ERR_INVALID),
    (dict(t=2 ** 24 + 1), pk.ERR_UNSUPPORTED), (dict(batch=0), pk.ERR_INVALID), (dict(batch=65536), pk.ERR_UNSUPPORTED),
    (dict(ws=0), pk.ERR_WORKSPACE), (dict(ws=FAKE + 128), pk.ERR_WORKSPACE), (dict(ws_bytes=1000), pk.ERR_WORKSPACE),
    (dict(pages=None), pk.ERR_INVALID), (dict(pages=_pages(n=0)), pk.ERR_INVALID), (dict(pages=_pages(K=FAKE + 4)), pk.ERR_INVALID)])
def test_paged_attend_refuses(change, code):
    a = dict(q=FAKE, qs=1024, pages=_pages(), table=FAKE, width=8, lens=FAKE, offsets=FAKE, counts=0, t=6, most=2, batch=3, scale=0.1,
             cap=0.0, slopes=0, out=FAKE, ws=FAKE, ws_bytes=1 << 28)
    a.update(change)
    assert pk.lib().pariskv_paged_attend(
        _cfg().c(), _vp(a["q"]), a["qs"], a["pages"], _vp(a["table"]), a["width"], _vp(a["lens"]), _vp(a["offsets"]), _vp(a["counts"]),
        a["t"], a["most"], a["batch"], ctypes.c_float(a["scale"]), ctypes.c_float(a["cap"]), _vp(a["slopes"]), _vp(a["out"]),
        _vp(a["ws"]), a["ws_bytes"], None) == code


def test_no_tokens_do_nothing():
    f = ctypes.c_float
    assert pk.lib().pariskv_paged_attend(_cfg().c(), None, 1024, _pages(), None, 8, None, None, None, 0, 1, 3, f(0.1), f(0), None, None,
                                         None, 0, None) == pk.OK
    assert pk.lib().pariskv_rotate_rows(_cfg().c(), _pages(), None, 1024, None, 256, None, 256, 0, None, None, None, 128, 0, None, None,
                                        f(0), None, None) == pk.OK


def test_workspace_sizes_grow_with_the_call():
    cfg = _cfg()
    sizes = [pk.paged_workspace_size(cfg, b, b * m, m) for b, m in ((1, 1), (8, 4), (8, 8), (8, 9), (64, 100), (64, 10000))]
    assert sizes == sorted(sizes) and sizes[0] >= 256 and sizes[-1] < 80 << 20 and all(x % 256 == 0 for x in sizes)
    assert pk.paged_workspace_size(cfg, 0, 4, 1) == pk.paged_workspace_size(cfg, 1, -1, 1) == 0
    assert pk.paged_workspace_size(cfg, 3, 0) == 256 and pk.paged_workspace_size(cfg, 1, 4, 0) == 0


def test_calls_of_too_many_blocks_are_refused():
    wide = pk.Config(64, 16, 1, workloads.rotation_signs(3))
    assert pk.paged_workspace_size(wide, 65535, 2 ** 24, 2 ** 20) == 0  # tiles of rows
    assert pk.paged_workspace_size(wide, 65535, 65535, 1) > 0


def _t(*shape, dtype=f16):
    return torch.zeros(shape, dtype=dtype)


def _cache(hkv=2, size=16):
    return pk.PagedCache(_t(10, hkv, size, 128), _t(10, hkv, size, 128))


@pytest.mark.parametrize("change,error,message", [
    ({}, ValueError, "must be a GPU tensor"), (dict(table=_t(2, dtype=i32)), ValueError, "table"), (dict(table=_t(2, 8)), TypeError, "table must be"),
    (dict(free=_t(10, 1, dtype=i32)), ValueError, "free"), (dict(n_free=_t(2, dtype=i32)), ValueError, "n_free must have shape"),
    (dict(lens=_t(3, dtype=i32)), ValueError, "lens must have shape"), (dict(counts=_t(2, dtype=torch.int64)), TypeError, "counts must be"),
    (dict(counts=None), ValueError, "counts is required"), (dict(t=None), ValueError, "t is required"), (dict(plan=3), TypeError, "PagePlan"),
    (dict(table=_t(2, 16, dtype=i32)[:, ::2]), ValueError, "table must be contiguous")])
def test_binding_refuses_plans(change, error, message):
    a = dict(table=_t(2, 8, dtype=i32), free=_t(10, dtype=i32), n_free=_t(1, dtype=i32), lens=_t(2, dtype=i32), counts=_t(2, dtype=i32), t=5,
             plan=pk.PagePlan.empty(2, 5, device="cpu"))
    if "t" in change or "plan" in change:
        a["plan"] = change.get("plan")
    a.update(change)
    with pytest.raises(error, match=message):
        pk.plan_pages(a["table"], a["free"], a["n_free"], a["lens"], a["counts"], 16, t=a["t"], plan=a["plan"])


@pytest.mark.parametrize("field,value,error", [
    ("lens", _t(3, dtype=i32), ValueError), ("offsets", _t(2, dtype=i32), ValueError), ("slots", _t(5), TypeError),
    ("positions", _t(4, dtype=i32), ValueError), ("counts", None, ValueError), ("slots", _t(5, 1, dtype=i32), ValueError)])
def test_binding_refuses_a_plans_arrays(field, value, error):
    plan = pk.PagePlan.empty(2, 5, device="cpu")
    setattr(plan, field, value)
    with pytest.raises(error, match=f"plan.{field}"):
        pk.plan_pages(_t(2, 8, dtype=i32), _t(10, dtype=i32), _t(1, dtype=i32), _t(2, dtype=i32), _t(2, dtype=i32), 16, plan=plan)


@pytest.mark.parametrize("change,error,message", [
    ({}, ValueError, "must be a GPU tensor"), (dict(q=_t(4, 1024)), ValueError, "q must be"), (dict(q=_t(4, 7, 128)), ValueError, "q must have shape"),
    (dict(k=_t(3, 2, 128)), ValueError, "k must have shape"), (dict(v=_t(4, 2, 128, dtype=f32)), TypeError, "v must be"),
    (dict(k=_t(4, 2, 256)[:, :, ::2]), ValueError, "next to each other"), (dict(k=_t(4, 4, 128)[:, ::2]), ValueError, "next to each other"),
    (dict(v=_t(4, 260)[:, :256].view(4, 2, 128)), ValueError, "multiple of 8"), (dict(cache=3), TypeError, "PagedCache"),
    (dict(cache=_cache(hkv=3)), ValueError, "cache.K must have shape"), (dict(cache=pk.PagedCache(_t(10, 2, 16, 128), _t(9, 2, 16, 128))),
                                                                         ValueError, "cache.V must have shape"),
    (dict(cache=pk.PagedCache(_t(10, 16, 256), None)), ValueError, "cache.K must be"),
    (dict(positions=_t(4, dtype=torch.int64)), TypeError, "positions must be"), (dict(slots=_t(5, dtype=i32)), ValueError, "slots must have"),
    (dict(freqs=_t(64)), TypeError, "freqs must be"), (dict(freqs=_t(8, 8, dtype=f32)), ValueError, "freqs must be"),
    (dict(q_weight=_t(64, dtype=f32)), ValueError, "q_weight must have"), (dict(k_weight=_t(128)), TypeError, "k_weight must be"),
    (dict(q_out=_t(4, 8, 64)), ValueError, "q_out must have")])
def test_binding_refuses_rows(change, error, message):
    a = dict(cache=_cache(), q=_t(4, 8, 128), k=_t(4, 2, 128), v=_t(4, 2, 128), positions=_t(4, dtype=i32), slots=_t(4, dtype=i32))
    a.update(change)
    args = [a.pop(x) for x in ("cache", "q", "k", "v", "positions", "slots")]
    with pytest.raises(error, match=message):
        pk.rotate_rows(_cfg(), *args, **a)


@pytest.mark.parametrize("change,error,message", [
    ({}, ValueError, "must be a GPU tensor"), (dict(q=_t(4, 9, 128)), ValueError, "q must have shape"), (dict(cache=None), TypeError, "PagedCache"),
    (dict(table=_t(3, dtype=i32)), ValueError, "table must be"), (dict(table=_t(3, 8)), TypeError, "table must be"),
    (dict(lens=_t(4, dtype=i32)), ValueError, "lens must have"), (dict(offsets=_t(3, dtype=i32)), ValueError, "offsets must have"),
    (dict(counts=_t(3)), TypeError, "counts must be"), (dict(slopes=_t(2, dtype=f32)), ValueError, "slopes must have"),
    (dict(out=_t(4, 8, 128, dtype=f32)), TypeError, "out must be"), (dict(out=_t(8, 8, 128)[::2]), ValueError, "out must be contiguous"),
    (dict(workspace=_t(512)), TypeError, "workspace must be"), (dict(workspace=_t(8, 8, dtype=u8)), ValueError, "workspace must have")])
def test_binding_refuses_attention(change, error, message):
    a = dict(q=_t(4, 8, 128), cache=_cache(), table=_t(3, 8, dtype=i32), lens=_t(3, dtype=i32), offsets=_t(4, dtype=i32))
    a.update(change)
    args = [a.pop(x) for x in ("q", "cache", "table", "lens", "offsets")]
    with pytest.raises(error, match=message):
        pk.paged_attend(_cfg(), *args, 0.1, **a)
