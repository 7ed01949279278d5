"""Scores of any finite size: a difference of two scores decides their weights, however large both are."""

import numpy as np
import pytest

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, draw, gpu
from oracle import quant

pytestmark = pytest.mark.gpu


def _cfg(hkv, g):
    return pk.Config(hkv, g, 64, workloads.rotation_signs(3))


def _want(q, K, V, visible, scale, half_out):
    """Outputs and their tolerance where the visible keys with the largest score, equal keys, have all the weight."""
    s = np.where(visible, scale * (q.astype(np.float64) @ K.astype(np.float64).T), -np.inf)
    top = s.max(1, keepdims=True)
    best = s == top
    # A score is off by at most (4 sqrt(128) 2^-24 + 2^-22) of A = |scale| sum |q k| (see tolerance()): a key that is both
    # its own and the top's such error and 30 below the top weighs less than e^-30.
    off = (4 * np.sqrt(128) * 2.0 ** -24 + 2.0 ** -22) * abs(scale) * (
        np.abs(q.astype(np.float64)) @ np.abs(K.astype(np.float64)).T)
    lowest = np.where(best, s - off, np.inf).min(1)
    clear = np.where(best, -np.inf, s + off).max(1) < lowest - 30
    assert clear.mean() > 0.9, "the inputs leave the choice open"
    w = best / best.sum(1, keepdims=True)
    return w @ V.astype(np.float64), (2.0 ** -19 + (2.0 ** -10 if half_out else 0.0)) * np.abs(V).max(), clear


def _check(got, q, K, V, visible, scale, half_out, what):
    want, tol, clear = _want(q, K, V, visible, scale, half_out)
    assert np.isfinite(got).all(), f"{what}: {(~np.isfinite(got)).sum()} values are not finite"
    off = np.abs(got.astype(np.float64) - want)[clear].max()
    assert off <= tol, f"{what}: off by {off:.3g}, allowed {tol:.3g}"


def _rows(r, b, hkv, n, size, order):
    """Keys of entries up to `size` times 4, each of them there twice (the same key in two places: equal scores);
    growing along the cache, shrinking, or in no order."""
    half = draw(r, b, hkv, (n + 1) // 2, D).clip(-4, 4)
    K = np.concatenate([half, half], 2)[:, :, r.permutation(2 * ((n + 1) // 2))[:n]].astype(np.float32)
    ramp = {"none": 1.0, "grows": np.linspace(0.02, 1, n)[:, None], "falls": np.linspace(1, 0.02, n)[:, None]}[order]
    return (K * ramp * size).astype(np.float16)


CASES = [(40.0, 16000.0, SCALE), (16000.0, 16000.0, SCALE), (16000.0, 16000.0, -1.0), (1.0, 1.0, 1e9)]


@pytest.mark.parametrize("order", ["none", "grows", "falls"])
@pytest.mark.parametrize("qsize,ksize,scale", CASES)
@pytest.mark.parametrize("g,t,n,bits", [(4, 3, 300, None), (4, 8, 3000, None), (4, 16, 3000, None), (4, 31, 3000, None),
                                        (4, 3, 3000, (8, 8)), (4, 8, 300, (4, 4)), (4, 31, 3000, (8, 8))])
def test_drafts(g, t, n, bits, qsize, ksize, scale, order):
    print(f"[large] drafts g {g} t {t} n {n} bits {bits} sizes {qsize} {ksize} scale {scale} {order}", flush=True)
    b, hkv = 1, 2
    r = np.random.default_rng(n + t)
    cfg = _cfg(hkv, g)
    K, V = _rows(r, b, hkv, n, ksize, order), draw(r, b, hkv, n, D)
    Kt, Vt = _rows(r, b, hkv, t, ksize, "none"), draw(r, b, hkv, t, D)
    q = (draw(r, b, hkv * g, t, D).clip(-4, 4).astype(np.float32) * qsize).astype(np.float16)
    if bits:
        cache = pk.QuantCache.empty(cfg, b, n, *bits)
        pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, n)
        K, V = quant.round_trip(K, bits[0]), quant.round_trip(V, bits[1])
        out = pk.quant_tree_attend(cfg, gpu(q), cache, gpu(Kt), gpu(Vt), n, scale).cpu().numpy()
    else:
        out = pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, scale).cpu().numpy()
    visible = np.concatenate([np.ones((t, n), bool), np.tril(np.ones((t, t), bool))], 1)
    got, qs, ks, vs = [], [], [], []
    for h in range(hkv * g):
        k_, v_ = np.concatenate([K[0, h // g], Kt[0, h // g]]), np.concatenate([V[0, h // g], Vt[0, h // g]])
        _check(out[0, h], q[0, h], k_, v_, visible, scale, False, f"head {h}")


@pytest.mark.parametrize("order", ["none", "grows", "falls"])
@pytest.mark.parametrize("qsize,ksize,scale", CASES)
@pytest.mark.parametrize("b,hkv,g,pos,t,sink,window", [
    (1, 1, 4, 3000, 4, 40, 2000), (1, 2, 4, 3000, 8, 40, 2000), (1, 1, 4, 3000, 31, 0, 2000),
    (1, 1, 2, 500, 300, 40, 100), (1, 1, 2, 3000, 1100, 4, 700)])
def test_windows(b, hkv, g, pos, t, sink, window, qsize, ksize, scale, order):
    print(f"[large] window g {g} pos {pos} t {t} sizes {qsize} {ksize} scale {scale} {order}", flush=True)
    r = np.random.default_rng(pos + t)
    n = pos + t
    K, V = _rows(r, b, hkv, n, ksize, order), draw(r, b, hkv, n, D)
    q = (draw(r, b, hkv * g, t, D).clip(-4, 4).astype(np.float32) * qsize).astype(np.float16)
    got = pk.sink_window_attend(_cfg(hkv, g), gpu(q), gpu(K), gpu(V), pos, sink, window, scale).cpu().numpy()
    p, j = np.arange(pos, n)[:, None], np.arange(n)[None]
    visible = (j <= p) & ((j < sink) | (j > p - window))
    for h in range(hkv * g):
        _check(got[0, h], q[0, h], K[0, h // g], V[0, h // g], visible, scale, True, f"head {h}")


@pytest.mark.parametrize("qsize,ksize,scale", CASES)
def test_listed_rows(qsize, ksize, scale):
    b, hkv, g, n, k = 1, 2, 4, 500, 200
    r = np.random.default_rng(3)
    cfg = _cfg(hkv, g)
    K, V = _rows(r, b, hkv, n, ksize, "none"), draw(r, b, hkv, n, D)
    q = (draw(r, b, hkv * g, D).clip(-4, 4).astype(np.float32) * qsize).astype(np.float16)
    idx = np.stack([np.sort(r.permutation(n)[:k]) for _ in range(hkv * g)]).reshape(b, hkv * g, k).astype(np.int32)
    cache = pk.QuantCache.empty(cfg, b, n)
    pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, n)
    K, V = quant.round_trip(K, 8), quant.round_trip(V, 8)
    out = pk.quant_attend(cfg, gpu(q), cache, gpu(idx), scale).cpu().numpy()
    for h in range(hkv * g):
        rows = idx[0, h]
        _check(out[0, h][None], q[0, h][None], K[0, h // g, rows], V[0, h // g, rows], np.ones((1, k), bool), scale,
               False, f"head {h}")


@pytest.mark.parametrize("order", ["none", "grows", "falls"])
@pytest.mark.parametrize("t", [3, 8, 16, 31, 1100])
def test_scores_far_below_zero(t, order):
    # Every score is negative and large: the weights are those of the least negative ones.
    print(f"[large] below zero t {t} {order}", flush=True)
    hkv, g, n = 2, 4, 2500
    r = np.random.default_rng(t)
    cfg = _cfg(hkv, g)
    K = -np.abs(_rows(r, 1, hkv, n + t, 12000.0, order)) - np.float16(2000)
    V = draw(r, 1, hkv, n + t, D)
    q = (np.abs(draw(r, 1, hkv * g, t, D).clip(-4, 4).astype(np.float32)) * 8000 + 100).astype(np.float16)
    see = np.concatenate([np.ones((t, n), bool), np.tril(np.ones((t, t), bool))], 1)
    outs = [(pk.sink_window_attend(cfg, gpu(q), gpu(K), gpu(V), n, 0, n + t, SCALE), True)]
    if t <= pk.MAX_TREE:
        Kt, Vt = (np.ascontiguousarray(x[:, :, n:]) for x in (K, V))
        outs.append((pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, SCALE), False))
    for out, half in outs:
        for h in range(hkv * g):
            _check(out.cpu().numpy()[0, h], q[0, h], K[0, h // g], V[0, h // g], see, SCALE, half, f"head {h}")
