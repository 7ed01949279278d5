"""Refusals of the quantised cache's and the several-token entry points, through the C ABI and the binding.
Nothing is launched: no GPU needed."""

import ctypes
import os

import pytest
import torch

import paper_2602_07721_amd as pk
import workloads

pytestmark = pytest.mark.skipif(not os.path.exists(pk.LIB_PATH), reason="library not built")

FAKE = 0x10000
f16, i32, u8 = torch.float16, torch.int32, torch.uint8


def _cfg(**kw):
    a = dict(n_kv_heads=2, q_per_kv=4, capacity=64, rot_signs=workloads.rotation_signs(3))
    a.update(kw)
    return pk.Config(**a)


def _vp(x):
    return ctypes.c_void_p(x)


def _cache(rec=FAKE, cap=100, kb=8, vb=8, host=0):
    return ctypes.byref(pk._QuantCache(rec, cap, kb, vb, host))


def _error():
    return pk.lib().pariskv_last_error().decode()


def test_record_bytes():
    sizes = {(8, 8): 272, (8, 4): 208, (4, 8): 208, (4, 4): 144}
    for (k, v), n in sizes.items():
        assert pk.QuantCache.record_bytes(k, v) == n
    for bad in ((16, 8), (8, 0), (4, 5), (-8, 8)):
        assert pk.lib().pariskv_quant_record_bytes(*bad) == 0
        with pytest.raises(ValueError, match="must each be 8 or 4"):
            pk.QuantCache.record_bytes(*bad)


@pytest.mark.parametrize("change,code", [
    (dict(cache=_cache(rec=0)), pk.ERR_INVALID), (dict(cache=_cache(rec=FAKE + 8)), pk.ERR_INVALID),
    (dict(cache=_cache(cap=0)), pk.ERR_INVALID), (dict(cache=_cache(cap=2 ** 30)), pk.ERR_INVALID),
    (dict(cache=_cache(kb=16)), pk.ERR_INVALID), (dict(cache=_cache(host=2)), pk.ERR_INVALID),
    (dict(cache=None), pk.ERR_INVALID), (dict(K=0), pk.ERR_INVALID), (dict(V=FAKE + 2), pk.ERR_INVALID),
    (dict(kv_cap=0), pk.ERR_INVALID), (dict(at=-1), pk.ERR_INVALID), (dict(at=41), pk.ERR_INVALID),
    (dict(t=-1), pk.ERR_INVALID), (dict(row=-1), pk.ERR_INVALID), (dict(row=91), pk.ERR_CAPACITY),
    (dict(rows=FAKE + 2), pk.ERR_INVALID), (dict(batch=0), pk.ERR_INVALID), (dict(batch=10000), pk.ERR_UNSUPPORTED),
    (dict(t=2 ** 27 + 1, kv_cap=2 ** 28, cache=_cache(cap=2 ** 28)), pk.ERR_UNSUPPORTED)])
def test_row_copies_refuse(change, code):
    a = dict(cache=_cache(), K=FAKE, V=FAKE, kv_cap=50, at=0, row=0, rows=0, t=10, batch=1)
    a.update(change)
    L, cfg = pk.lib(), _cfg()
    assert L.pariskv_quantize_rows(cfg.c(), a["cache"], _vp(a["K"]), _vp(a["V"]), a["kv_cap"], a["at"], a["row"],
                                   _vp(a["rows"]), a["t"], a["batch"], None) == code
    assert L.pariskv_dequantize_rows(cfg.c(), a["cache"], a["row"], _vp(a["rows"]), a["t"], _vp(a["K"]), _vp(a["V"]),
                                     a["kv_cap"], a["at"], a["batch"], None) == code


def test_no_rows_and_no_tokens_do_nothing():
    L, cfg = pk.lib(), _cfg()
    assert L.pariskv_quantize_rows(cfg.c(), _cache(), _vp(FAKE), _vp(FAKE), 50, 50, 100, None, 0, 1, None) == pk.OK
    assert L.pariskv_dequantize_rows(cfg.c(), _cache(), 100, None, 0, _vp(FAKE), _vp(FAKE), 50, 50, 1, None) == pk.OK
    f = ctypes.c_float(0.1)
    assert L.pariskv_tree_attend(cfg.c(), None, _vp(FAKE), _vp(FAKE), 100, None, None, None, 10, None, 0, 1, f, None, None,
                                 0, None) == pk.OK
    assert L.pariskv_sink_window_attend(cfg.c(), None, _vp(FAKE), _vp(FAKE), 100, 5, None, 0, None, 4, 8, 1, f, None, None,
                                        0, None) == pk.OK


@pytest.mark.parametrize("change,code", [
    (dict(k=0), pk.ERR_INVALID), (dict(k=4097), pk.ERR_UNSUPPORTED), (dict(q=0), pk.ERR_INVALID),
    (dict(out=FAKE + 4), pk.ERR_INVALID), (dict(idx=FAKE + 2), pk.ERR_INVALID), (dict(scale=float("inf")), pk.ERR_INVALID),
    (dict(cache=_cache(vb=3)), pk.ERR_INVALID), (dict(batch=0), pk.ERR_INVALID)])
def test_quant_attend_refuses(change, code):
    a = dict(q=FAKE, cache=_cache(), idx=FAKE, k=8, batch=1, scale=0.1, out=FAKE)
    a.update(change)
    L, cfg, win = pk.lib(), _cfg(), pk.Window(2, 2, 50, 60)
    rest = (a["cache"], _vp(a["idx"]), a["k"])
    tail = (a["batch"], ctypes.c_float(a["scale"]), _vp(a["out"]), None)
    assert L.pariskv_quant_attend(cfg.c(), _vp(a["q"]), *rest, *tail) == code
    assert L.pariskv_quant_tiered_attend(cfg.c(), _vp(a["q"]), _vp(FAKE), _vp(FAKE), 20, *rest, win.c(), *tail) == code


@pytest.mark.parametrize("win,wcap,kw,code", [
    (None, 20, FAKE, pk.ERR_INVALID), (pk.Window(2, 2, 50, 60), 11, FAKE, pk.ERR_INVALID),
    (pk.Window(2, 1, 50, 60), 20, FAKE, pk.ERR_INVALID), (pk.Window(2, 2, 50, 60), 0, FAKE, pk.ERR_INVALID),
    (pk.Window(2, 2, 50, 60), 20, 0, pk.ERR_INVALID), (pk.Window(0, 0, 50, 4143), 5000, FAKE, pk.ERR_UNSUPPORTED)])
def test_quant_tiered_attend_refuses_windows(win, wcap, kw, code):
    L, cfg = pk.lib(), _cfg()
    assert L.pariskv_quant_tiered_attend(cfg.c(), _vp(FAKE), _vp(kw), _vp(FAKE), wcap, _cache(), _vp(FAKE), 8,
                                         None if win is None else win.c(), 1, ctypes.c_float(0.1), _vp(FAKE),
                                         None) == code


@pytest.mark.parametrize("change,code", [
    (dict(t=65), pk.ERR_UNSUPPORTED), (dict(t=-1), pk.ERR_INVALID), (dict(n=-1), pk.ERR_INVALID),
    (dict(n=101), pk.ERR_INVALID), (dict(n=2 ** 30), pk.ERR_INVALID), (dict(q=0), pk.ERR_INVALID),
    (dict(out=FAKE + 8), pk.ERR_INVALID), (dict(kt=0), pk.ERR_INVALID), (dict(mask=FAKE + 4), pk.ERR_INVALID),
    (dict(lens=FAKE + 1), pk.ERR_INVALID), (dict(scale=float("nan")), pk.ERR_INVALID), (dict(ws=0), pk.ERR_WORKSPACE),
    (dict(ws=FAKE + 128), pk.ERR_WORKSPACE), (dict(ws_bytes=255), pk.ERR_WORKSPACE), (dict(batch=0), pk.ERR_INVALID)])
def test_tree_attend_refuses(change, code):
    a = dict(q=FAKE, kt=FAKE, mask=0, n=100, lens=0, t=4, batch=1, scale=0.1, out=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update(change)
    L, cfg = pk.lib(), _cfg()
    rest = (_vp(a["kt"]), _vp(FAKE), _vp(a["mask"]), a["n"], _vp(a["lens"]), a["t"], a["batch"],
            ctypes.c_float(a["scale"]), _vp(a["out"]), _vp(a["ws"]), a["ws_bytes"], None)
    assert L.pariskv_tree_attend(cfg.c(), _vp(a["q"]), _vp(FAKE), _vp(FAKE), 100, *rest) == code
    assert L.pariskv_quant_tree_attend(cfg.c(), _vp(a["q"]), _cache(), *rest) == code


def test_tree_attend_refuses_caches():
    L, cfg = pk.lib(), _cfg()
    rest = (_vp(FAKE), _vp(FAKE), None, 10, None, 4, 1, ctypes.c_float(0.1), _vp(FAKE), _vp(FAKE), 1 << 20, None)
    for K, V, cap in ((0, FAKE, 100), (FAKE, FAKE + 8, 100), (FAKE, FAKE, 0), (FAKE, FAKE, 2 ** 30)):
        assert L.pariskv_tree_attend(cfg.c(), _vp(FAKE), _vp(K), _vp(V), cap, *rest) == pk.ERR_INVALID
    assert L.pariskv_quant_tree_attend(cfg.c(), _vp(FAKE), None, *rest) == pk.ERR_INVALID
    assert L.pariskv_quant_tree_attend(cfg.c(), _vp(FAKE), _cache(host=1), *rest) == pk.ERR_UNSUPPORTED
    assert "device memory" in _error()


@pytest.mark.parametrize("change,code", [
    (dict(pos=-1), pk.ERR_INVALID), (dict(t=-1), pk.ERR_INVALID), (dict(pos=97), pk.ERR_INVALID),
    (dict(pos=2 ** 30, cap=2 ** 30 - 1), pk.ERR_INVALID), (dict(sink=-1), pk.ERR_INVALID), (dict(window=0), pk.ERR_INVALID),
    (dict(cap=0), pk.ERR_INVALID), (dict(cap=2 ** 30), pk.ERR_INVALID), (dict(scale=float("inf")), pk.ERR_INVALID),
    (dict(q=0), pk.ERR_INVALID), (dict(K=FAKE + 8), pk.ERR_INVALID), (dict(out=0), pk.ERR_INVALID),
    (dict(starts=FAKE + 2), pk.ERR_INVALID), (dict(counts=FAKE + 2), pk.ERR_INVALID), (dict(ws=0), pk.ERR_WORKSPACE),
    (dict(ws_bytes=0), pk.ERR_WORKSPACE), (dict(batch=0), pk.ERR_INVALID),
    (dict(batch=8000, pos=0, t=262 * 128 + 1, cap=2 ** 29), pk.ERR_UNSUPPORTED)])
def test_sink_window_attend_refuses(change, code):
    a = dict(q=FAKE, K=FAKE, cap=100, pos=96, starts=0, t=4, counts=0, sink=4, window=32, batch=1, scale=0.1, out=FAKE,
             ws=FAKE, ws_bytes=1 << 20)
    a.update(change)
    L, cfg = pk.lib(), _cfg()
    assert L.pariskv_sink_window_attend(
        cfg.c(), _vp(a["q"]), _vp(a["K"]), _vp(FAKE), a["cap"], a["pos"], _vp(a["starts"]), a["t"], _vp(a["counts"]),
        a["sink"], a["window"], a["batch"], ctypes.c_float(a["scale"]), _vp(a["out"]), _vp(a["ws"]), a["ws_bytes"],
        None) == code


def test_workspace_sizes():
    cfg = _cfg()
    assert pk.tree_workspace_size(cfg, 1, 100, 65) == 0 and pk.tree_workspace_size(cfg, 1, -1, 4) == 0
    assert pk.sink_window_workspace_size(cfg, 1, 0, 4, 0, 0) == 0
    for n in (0, 1, 100, 4096, 1 << 20, 2 ** 30 - 1):
        for t in (0, 1, 7, 64):
            size = pk.tree_workspace_size(cfg, 3, n, t)
            assert size >= 256 and size % 256 == 0
    for pos, t, window in ((0, 1, 1), (5000, 1, 4096), (5000, 1000, 4096), (0, 100000, 4096), (10, 0, 5)):
        size = pk.sink_window_workspace_size(cfg, 3, pos, t, 128, window)
        assert size >= 256 and size % 256 == 0


def _t(*shape, dtype=f16):
    return torch.zeros(shape, dtype=dtype)


def _rows_call(name, **change):
    a = dict(cache=pk.QuantCache(_t(1, 2, 100, 272, dtype=u8)), K=_t(1, 2, 50, 128), V=_t(1, 2, 50, 128), row=0)
    a.update(change)
    if name == "quantize_rows":
        return pk.quantize_rows(_cfg(), a["cache"], a["K"], a["V"], 0, a["row"], 4)
    return pk.dequantize_rows(_cfg(), a["cache"], a["row"], 4, a["K"], a["V"])


@pytest.mark.parametrize("name", ["quantize_rows", "dequantize_rows"])
@pytest.mark.parametrize("change,error,message", [
    ({}, ValueError, "K must be a GPU tensor"), (dict(K=_t(2, 50, 128)), ValueError, "K must be"),
    (dict(K=_t(1, 3, 50, 128)), ValueError, "K must have shape"), (dict(V=_t(1, 2, 49, 128)), ValueError, "V must have shape"),
    (dict(V=None), ValueError, "V is required"), (dict(K=_t(1, 2, 50, 128, dtype=torch.bfloat16)), TypeError, "K must be"),
    (dict(K=_t(1, 2, 100, 128)[:, :, ::2]), ValueError, "K must be contiguous"), (dict(cache=3), TypeError, "QuantCache"),
    (dict(cache=pk.QuantCache(_t(1, 2, 100, 208, dtype=u8))), ValueError, "cache.rec must have shape"),
    (dict(cache=pk.QuantCache(_t(1, 2, 100, 272))), TypeError, "cache.rec must be"),
    (dict(cache=pk.QuantCache(_t(1, 2, 100, 272, dtype=u8), host_mapped=True)), ValueError, "pinned"),
    (dict(row=_t(2, dtype=i32)), ValueError, "row must have shape"), (dict(row=_t(1)), TypeError, "row must be")])
def test_binding_refuses_rows(name, change, error, message):
    with pytest.raises(error, match=message):
        _rows_call(name, **change)


@pytest.mark.parametrize("change,error,message", [
    ({}, ValueError, "must be a GPU tensor"), (dict(q=_t(1, 8, 128)), ValueError, "q must be"),
    (dict(q=_t(1, 8, 4, 64)), ValueError, "q must have shape"), (dict(K_tree=_t(1, 2, 5, 128)), ValueError, "K_tree must have"),
    (dict(V_tree=_t(1, 8, 4, 128)), ValueError, "V_tree must have"), (dict(mask=_t(1, 4, dtype=i32)), TypeError, "mask must be"),
    (dict(mask=_t(1, 5, dtype=torch.int64)), ValueError, "mask must have"), (dict(lens=_t(2, dtype=i32)), ValueError, "lens must have"),
    (dict(out=_t(1, 8, 4, 128)), TypeError, "out must be"), (dict(workspace=_t(8, 8, dtype=u8)), ValueError, "workspace must have"),
    (dict(q=_t(1, 8, 8, 128)[:, :, ::2]), ValueError, "q must be contiguous")])
def test_binding_refuses_trees(change, error, message):
    a = dict(q=_t(1, 8, 4, 128), K_tree=_t(1, 2, 4, 128), V_tree=_t(1, 2, 4, 128))
    a.update(change)
    q, Kt, Vt = a.pop("q"), a.pop("K_tree"), a.pop("V_tree")
    with pytest.raises(error, match=message):
        pk.tree_attend(_cfg(), q, _t(1, 2, 50, 128), _t(1, 2, 50, 128), Kt, Vt, 10, 0.1, **a)
    with pytest.raises(error, match=message):
        pk.quant_tree_attend(_cfg(), q, pk.QuantCache(_t(1, 2, 50, 272, dtype=u8)), Kt, Vt, 10, 0.1, **a)


@pytest.mark.parametrize("change,error,message", [
    ({}, ValueError, "must be a GPU tensor"), (dict(q=_t(1, 8, 128)), ValueError, "q must be"),
    (dict(K=_t(2, 2, 50, 128)), ValueError, "K must have"), (dict(V=_t(1, 2, 51, 128)), ValueError, "V must have"),
    (dict(starts=_t(1, dtype=torch.int64)), TypeError, "starts must be"), (dict(counts=_t(2, dtype=i32)), ValueError, "counts must have"),
    (dict(out=_t(1, 8, 4, 128, dtype=torch.float32)), TypeError, "out must be"),
    (dict(workspace=_t(512)), TypeError, "workspace must be")])
def test_binding_refuses_windows(change, error, message):
    a = dict(q=_t(1, 8, 4, 128), K=_t(1, 2, 50, 128), V=_t(1, 2, 50, 128))
    a.update(change)
    q, K, V = a.pop("q"), a.pop("K"), a.pop("V")
    with pytest.raises(error, match=message):
        pk.sink_window_attend(_cfg(), q, K, V, 10, 4, 16, 0.1, **a)


def test_binding_refuses_quant_attend():
    cfg, q, idx = _cfg(), _t(1, 8, 128), _t(1, 8, 16, dtype=i32)
    cache = pk.QuantCache(_t(1, 2, 50, 272, dtype=u8))
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        pk.quant_attend(cfg, q, cache, idx, 0.1)
    with pytest.raises(ValueError, match="idx must have shape"):
        pk.quant_attend(cfg, q, cache, _t(1, 7, 16, dtype=i32), 0.1)
    with pytest.raises(TypeError, match="QuantCache"):
        pk.quant_attend(cfg, q, q, idx, 0.1)
    with pytest.raises(ValueError, match="K_win must have shape"):
        pk.quant_tiered_attend(cfg, q, _t(1, 3, 20, 128), _t(1, 3, 20, 128), cache, idx, pk.Window(0, 0, 50, 60), 0.1)
