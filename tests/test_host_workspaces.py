"""A workspace sized for the largest call serves every smaller one.  Nothing is launched: no GPU needed."""

import ctypes
import os
import random
import re

import pytest

import paper_2602_07721_amd as pk
import workloads

pytestmark = pytest.mark.skipif(not os.path.exists(pk.LIB_PATH), reason="library not built")

FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced: a workspace of 0 bytes is refused before any launch


def _cfg(hkv, g):
    return pk.Config(hkv, g, 64, workloads.rotation_signs(3))


def _refused():
    found = re.search(r"workspace has 0 bytes, needs (\d+)", pk.lib().pariskv_last_error().decode())
    assert found, pk.lib().pariskv_last_error()
    return int(found.group(1))


def _tree_need(cfg, batch, n, t):
    rc = pk.lib().pariskv_tree_attend(cfg.c(), FAKE, FAKE, FAKE, max(1, n), FAKE, FAKE, None, n, None, t, batch,
                                      ctypes.c_float(0.1), FAKE, FAKE, 0, None)
    assert rc == pk.ERR_WORKSPACE
    return _refused()


def _window_need(cfg, batch, pos, t, sink, window):
    rc = pk.lib().pariskv_sink_window_attend(cfg.c(), FAKE, FAKE, FAKE, pos + t, pos, None, t, None, sink, window, batch,
                                             ctypes.c_float(0.1), FAKE, FAKE, 0, None)
    assert rc == pk.ERR_WORKSPACE
    return _refused()


def _log(rng, lo, hi):
    return min(hi, max(lo, int(lo * (hi / lo) ** rng.random() + 0.5)))


@pytest.mark.parametrize("hkv,g", [(1, 1), (1, 8), (2, 5), (8, 4), (4, 7), (3, 16), (40, 2)])
def test_drafts(hkv, g):
    rng, cfg = random.Random(hkv * 100 + g), _cfg(hkv, g)
    for _ in range(60):
        batch, n, t = _log(rng, 1, 64), _log(rng, 1, 1 << 20), rng.randint(1, 64)
        size = pk.tree_workspace_size(cfg, batch, n, t)
        assert size >= _tree_need(cfg, batch, n, t)
        for _ in range(60):
            b_, n_, t_ = rng.randint(1, batch), rng.choice([n, n, rng.randint(0, n)]), rng.randint(1, t)
            n_ = max(0, n_ - rng.randint(0, 300))
            need = _tree_need(cfg, b_, n_, t_)
            assert need <= size, f"batch {b_} n {n_} t {t_} needs {need}, batch {batch} n {n} t {t} has {size}"
            assert pk.tree_workspace_size(cfg, b_, n_, t_) <= size


@pytest.mark.parametrize("hkv,g", [(1, 1), (1, 8), (2, 5), (8, 4), (4, 7), (3, 16), (40, 2)])
def test_windows(hkv, g):
    rng, cfg = random.Random(hkv * 100 + g), _cfg(hkv, g)
    for _ in range(60):
        batch, pos, t = _log(rng, 1, 64), _log(rng, 1, 1 << 17), _log(rng, 1, 8192)
        sink, window = rng.choice([0, 4, 128]), _log(rng, 1, 1 << 17)
        size = pk.sink_window_workspace_size(cfg, batch, pos, t, sink, window)
        assert size >= _window_need(cfg, batch, pos, t, sink, window)
        for _ in range(60):
            b_, p_ = rng.randint(1, batch), max(0, rng.choice([pos, pos, rng.randint(0, pos)]) - rng.randint(0, 300))
            t_, s_, w_ = _log(rng, 1, t), rng.choice([sink, sink // 2]), rng.choice([window, window, rng.randint(1, window)])
            need = _window_need(cfg, b_, p_, t_, s_, w_)
            assert need <= size, f"{(b_, p_, t_, s_, w_)} needs {need}, {(batch, pos, t, sink, window)} has {size}"
            assert pk.sink_window_workspace_size(cfg, b_, p_, t_, s_, w_) <= size


def test_sizes_that_once_fell():
    cfg = _cfg(8, 4)
    for long, short in ((16448, 16320), (16512, 16384), (65568, 65536), (32800, 32768)):
        assert pk.tree_workspace_size(cfg, 1, long, 8) >= _tree_need(cfg, 1, short, 8)
    assert pk.sink_window_workspace_size(cfg, 1, 4096, 507, 4, 4096) >= _window_need(cfg, 1, 4096, 480, 4, 4096)
    assert pk.sink_window_workspace_size(cfg, 1, 5000, 4096, 128, 4096) >= _window_need(cfg, 1, 5000, 1, 128, 4096)


def test_sizes_stay_small():
    # About two rounds of blocks, each with a float32 state of its rows: never more than 70 MB, whatever the sizes.
    for hkv, g in ((1, 1), (8, 4), (3, 16), (64, 8)):
        cfg = _cfg(hkv, g)
        assert pk.tree_workspace_size(cfg, 64, 2 ** 30 - 1, 64) <= 70 << 20
        assert pk.sink_window_workspace_size(cfg, 64, 2 ** 29, 2 ** 14, 128, 2 ** 29) <= 70 << 20
