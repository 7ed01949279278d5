"""Infinities and NaNs in values that every token sees leave their dims not finite, and all others as they are."""

import numpy as np
import pytest

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, attend64, check, draw, gpu, tolerance

pytestmark = pytest.mark.gpu

BAD = {3: np.inf, 64: -np.inf, 127: np.nan}  # by dim


def _cfg(hkv, g):
    return pk.Config(hkv, g, 64, workloads.rotation_signs(3))


def _spoil(V, rows):
    """V with such a value in each of the rows, a dim of its own each; and which dims those are."""
    bad, dims = V.copy(), []
    for i, (row, (dim, x)) in enumerate(zip(rows, BAD.items())):
        bad[:, :, row, dim] = x
        V[:, :, row, dim] = 0
        dims.append(dim)
    return bad, np.isin(np.arange(D), dims)


def _compare(got, q, K, V, visible, hit, half_out, what):
    assert not np.isfinite(got[:, hit]).any(), f"{what}: finite where a value is not"
    want = attend64(q, K, V, visible)
    check(got[:, ~hit], want[:, ~hit], tolerance(q, K, V, half_out=half_out), what)


@pytest.mark.parametrize("g,t", [(4, 1), (4, 8), (4, 16), (4, 31)])
@pytest.mark.parametrize("n", [70, 3001])
def test_cached_rows_of_drafts(g, t, n):
    print(f"[not finite] drafts g {g} t {t} n {n}", flush=True)
    b, hkv = 2, 2
    r = np.random.default_rng(n + t)
    K, V, q = draw(r, b, hkv, n, D), draw(r, b, hkv, n, D), draw(r, b, hkv * g, t, D)
    Kt, Vt = draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    bad, hit = _spoil(V, (0, n // 2, n - 1))
    out = pk.tree_attend(_cfg(hkv, g), gpu(q), gpu(K), gpu(bad), gpu(Kt), gpu(Vt), n, SCALE).cpu().numpy()
    visible = np.concatenate([np.ones((t, n), bool), np.tril(np.ones((t, t), bool))], 1)
    for s in range(b):
        for h in range(hkv * g):
            k_, v_ = np.concatenate([K[s, h // g], Kt[s, h // g]]), np.concatenate([V[s, h // g], Vt[s, h // g]])
            _compare(out[s, h], q[s, h], k_, v_, visible, hit, False, f"seq {s} head {h}")


@pytest.mark.parametrize("b,hkv,g,pos,t,sink,window", [
    (1, 1, 4, 3000, 1, 40, 2000), (1, 2, 4, 3000, 8, 40, 2000), (1, 1, 4, 3000, 16, 40, 2000),
    (1, 1, 4, 3000, 40, 40, 2000), (1, 2, 2, 3000, 300, 40, 2000), (1, 1, 2, 3000, 1100, 70, 2000)])
def test_rows_inside_every_window(b, hkv, g, pos, t, sink, window):
    print(f"[not finite] window g {g} pos {pos} t {t}", flush=True)
    r = np.random.default_rng(pos + t)
    n = pos + t
    K, V, q = draw(r, b, hkv, n, D), draw(r, b, hkv, n, D), draw(r, b, hkv * g, t, D)
    bad, hit = _spoil(V, (pos - 200, pos - 201, 7))  # two rows inside every window and a sink
    got = pk.sink_window_attend(_cfg(hkv, g), gpu(q), gpu(K), gpu(bad), pos, sink, window, SCALE).cpu().numpy()
    p, j = np.arange(pos, n)[:, None], np.arange(n)[None]
    visible = (j <= p) & ((j < sink) | (j > p - window))
    for h in range(hkv * g):
        _compare(got[0, h], q[0, h], K[0, h // g], V[0, h // g], visible, hit, True, f"head {h}")
