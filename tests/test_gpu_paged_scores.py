"""Scores of the attention over pages at the ends of their range: caps, keys that a token does not attend, factors."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
from new_tokens import D, SCALE, check, gpu
from pages import Pool, attend64, config, ints, tolerance

pytestmark = pytest.mark.gpu


def _set_key(pool, b, row, k):
    pool.rows[b][0][row] = k
    pool.K[pool.table[b, row // pool.page], :, row % pool.page] = k


def _run(pool, q, offsets, hkv, g, cap, slopes=None, scale=SCALE, most=None):
    return pk.paged_attend(config(hkv, g), gpu(q), pool.cache(), ints(pool.table), ints(pool.lens), ints(offsets), scale,
                           max_tokens=int(max(np.diff(offsets))) if most is None else most, softcap=cap,
                           slopes=None if slopes is None else gpu(slopes)).cpu().numpy()


def _fine(q, k, v, slopes):
    """tolerance() without the term of the cap, for scores far below it: there a capped score is a series, off by four
    roundings to float32 of itself, which a weight is off by and an output twice."""
    A = SCALE * (np.abs(q.astype(np.float64)).reshape(-1, D) @ np.abs(k.astype(np.float64)).T).max()
    return tolerance(q, k, v, SCALE, 0.0, slopes) + 2 * 4 * 2.0 ** -24 * A * np.abs(v.astype(np.float64)).max()


# 16 and 32 rows a wave, tiles of rows.
@pytest.mark.parametrize("m,g", [(4, 4), (8, 4), (60, 2)])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("who", ["later key", "other head"])
def test_large_scores_that_a_row_has_no_part_in_leave_it_alone(m, g, bias, who):
    # A cap of 2^20, scores of a few units, and some of more than 2^18: of a key behind the token, or of another head.
    cap, n = 2.0 ** 20, 200
    print(f"[paged] {m} tokens g {g} bias {bias} large scores of a {who}", flush=True)
    r = np.random.default_rng(m)
    pool = Pool(r, 1, [n], 16)
    q = r.standard_normal((m, g, D)).astype(np.float16)
    rows = slice(0, m)
    if who == "later key":
        _set_key(pool, 0, n - 1, np.full(D, 60000, np.float16))
        q = np.abs(q) + np.float16(0.25)  # its scores: above 0.088 x 60000 x 128 / 4
        rows = slice(0, m - 1)
    else:
        q[:, 1] = np.where(np.arange(D) % 2 == 0, 60000, 30000)
        _set_key(pool, 0, n // 2, np.full(D, 8, np.float16))  # 0.088 x 8 x 45000 x 128
    slopes = np.linspace(0.01, 0.2, g).astype(np.float32) if bias else None
    got = _run(pool, q, [0, m], 1, g, cap, slopes)
    k, v = (x[:, 0] for x in pool.rows[0])
    p = np.arange(n - m, n)[rows]
    heads = [h for h in range(g) if who == "later key" or h != 1]
    seen = k[:n - 1] if who == "later key" else k
    sl = None if slopes is None else slopes[heads]
    want = attend64(q[rows][:, heads], k, v, p, np.ones(n, bool), SCALE, cap, sl)
    check(got[rows][:, heads], want, _fine(q[rows][:, heads], seen, v, sl), who)


# Scores on both sides of a fifth of the cap in the same wave; caps on both sides of 64, where their form changes.
@pytest.mark.parametrize("cap", [64.0, 64.5, 100.0, 1000.0])
@pytest.mark.parametrize("m,g", [(1, 4), (8, 4), (60, 2)])
@pytest.mark.parametrize("bias", [False, True])
def test_caps_on_both_sides_of_the_change_of_form(cap, m, g, bias):
    n, law = 333, (4.0 * cap / 64.0) ** 0.5 if cap > 64.5 else 4.0
    print(f"[paged] cap {cap} {m} tokens g {g} bias {bias}", flush=True)
    r = np.random.default_rng(m + int(cap))
    pool = Pool(r, 1, [n], 16, law=law)
    q = (law * r.standard_normal((m, g, D))).astype(np.float16)
    slopes = np.linspace(0.01, 0.2, g).astype(np.float32) if bias else None
    got = _run(pool, q, [0, m], 1, g, cap, slopes)
    k, v = (x[:, 0] for x in pool.rows[0])
    want = attend64(q, k, v, np.arange(n - m, n), np.ones(n, bool), SCALE, cap, slopes)
    check(got, want, tolerance(q, k, v, SCALE, cap, slopes), f"cap {cap}")


@pytest.mark.parametrize("m,g", [(1, 4), (8, 4), (60, 2)])
@pytest.mark.parametrize("scale,cap,slope", [(3e38, 0.0, None), (-3e38, 0.0, None), (3e38, 0.0, 0.5), (1e37, 2.0 ** -20, None),
                                             (1e37, 2.0 ** -20, 0.25), (SCALE, 0.0, 3e38)])
def test_factors_past_the_largest_float32(m, g, scale, cap, slope):
    # Finite scales, slopes and scores, whose factors log2(e) scale, scale / softcap and log2(e) slope are not.  Products
    # of query and key are 2^-20 times whole numbers, so without a cap scores are alike or so far apart that all weight
    # lies on the largest; with it they are -cap, 0 and cap.  What is left is the roundings of weights and outputs.
    n = 90
    print(f"[paged] scale {scale} cap {cap} slope {slope} {m} tokens g {g}", flush=True)
    r = np.random.default_rng(m)
    pool = Pool(r, 1, [n], 16)
    for j in range(n):
        k = np.zeros(D, np.float16)
        k[0] = r.integers(-3, 4) / 1024
        _set_key(pool, 0, j, k)
    q = np.zeros((m, g, D), np.float16)
    q[:, :, 0] = r.choice([-1, 1], (m, g)) / 1024
    slopes = None if slope is None else np.full(g, slope, np.float32)
    got = _run(pool, q, [0, m], 1, g, cap, slopes, scale=scale)
    k, v = (x[:, 0] for x in pool.rows[0])
    want = attend64(q, k, v, np.arange(n - m, n), np.ones(n, bool), scale, cap, slopes)
    rel = 2.0 ** -10 + 2.0 ** -19 + (2 * 2.0 ** -21 * cap if cap else 0.0)
    if cap and slope:  # biases to slope n, rounded with their sum: see tolerance()
        rel += 2 * 2.0 ** -23 * (2 * cap + 40 + cap)
    check(got, want, rel * np.abs(v.astype(np.float64)).max(), f"scale {scale}")


@pytest.mark.parametrize("m", [1, 40])
def test_dense_forms_take_the_same_scales(m):
    r = np.random.default_rng(m)
    n, g = 90, 4
    K = np.zeros((1, 1, n, D), np.float16)
    K[..., 0] = r.integers(-3, 4, n) / 1024
    V = r.standard_normal((1, 1, n, D)).astype(np.float16)
    q = np.zeros((1, g, m, D), np.float16)
    q[..., 0] = r.choice([-1, 1], (g, m)) / 1024
    got = pk.sink_window_attend(config(1, g), gpu(q), gpu(K), gpu(V), n - m, 0, n, 3e38).cpu().numpy()
    want = attend64(q[0].transpose(1, 0, 2), K[0, 0], V[0, 0], np.arange(n - m, n), np.ones(n, bool), 3e38, 0.0, None)
    check(got[0].transpose(1, 0, 2), want, (2.0 ** -10 + 2.0 ** -19) * np.abs(V.astype(np.float64)).max(), f"{m} tokens")
