"""Few new tokens over pages: reads past the caches, several heads and long sequences; and what the walk promises of its
weights, which float16 outputs near the largest value would not show."""

import numpy as np
import pytest

import paper_2602_07721_amd as pk
from new_tokens import D, SCALE, check, gpu
from pages import Pool, attend64, config, ints, tolerance

pytestmark = pytest.mark.gpu

HKV, G, PAGE = 8, 4, 16
LENS = [60000, 3000, 129]
# From 192 MB on, parts of 128 keys of one KV head at 64 KB, keys and values are read past the caches.
STREAMED = (192 << 20) // (64 << 10)


@pytest.fixture(scope="module")
def pool():
    assert sum(-(-n // 128) for n in LENS) * HKV > STREAMED
    return Pool(np.random.default_rng(1), HKV, LENS, PAGE)


# Single tokens (16 rows a wave), 8 (32 rows, keys through the caches), and single tokens beside a chunk.
@pytest.mark.parametrize("counts", [[1, 1, 1], [8, 8, 8], [1, 1, 100]])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (20.0, True), (200.0, True)])
@pytest.mark.parametrize("lost", [False, True])
def test_calls_that_read_past_the_caches(pool, counts, cap, bias, lost):
    print(f"[paged] counts {counts} cap {cap} bias {bias} lost pages {lost}", flush=True)
    if counts[2] == 100:  # the walk has the first two alone
        assert sum(-(-n // 128) for n in LENS[:2]) * HKV > STREAMED
    r = np.random.default_rng(2)
    offsets = np.concatenate(([0], np.cumsum(counts)))
    q = r.standard_normal((int(offsets[-1]), HKV * G, D)).astype(np.float16)
    slopes = np.geomspace(0.5, 2.0 ** -10, HKV * G).astype(np.float32) if bias else None
    table, gone = pool.table.copy(), [(0, 7), (0, 1800), (0, 1801), (0, 3740), (1, 100)] if lost else []
    for b, j in gone:
        table[b, j] = -1
    got = pk.paged_attend(config(HKV, G), gpu(q), pool.cache(), ints(table), ints(LENS), ints(offsets), SCALE,
                          max_tokens=max(counts), softcap=cap, slopes=None if slopes is None else gpu(slopes)).cpu().numpy()
    for b, (n, m) in enumerate(zip(LENS, counts)):
        there = ~np.isin(np.arange(n) // PAGE, [j for s, j in gone if s == b])
        for h in (0, HKV - 1):
            k, v = (x[:, h] for x in pool.rows[b])
            qh = q[offsets[b]:offsets[b + 1]].reshape(m, HKV, G, D)[:, h]
            sl = None if slopes is None else slopes[h * G:(h + 1) * G]
            want = attend64(qh, k, v, np.arange(n - m, n), there, SCALE, cap, sl)
            check(got[offsets[b]:offsets[b + 1]].reshape(m, HKV, G, D)[:, h], want, tolerance(qh, k, v, SCALE, cap, sl),
                  f"seq {b} head {h}")


# most: of the call; with 100 its few rows are walked beside tiles.
@pytest.mark.parametrize("m,g,most", [(1, 4, 1), (4, 4, 4), (8, 4, 8), (2, 16, 2), (4, 4, 100)])
@pytest.mark.parametrize("n", [4, 20, 200, 5000])
def test_weights_keep_their_low_bits(m, g, most, n):
    # Keys in pairs whose weights differ, values that all but cancel: an output of a thousandth of the largest value, whose
    # own rounding hides little.  Scores are exact.  Weights rounded to float16 would be off by 2^-12 each.
    print(f"[paged] {m} tokens g {g} most {most} over {n} keys and their own", flush=True)
    r = np.random.default_rng(n + m)
    rows = n + m
    pool = Pool(r, 1, [rows], 16)
    steps = r.integers(-24, 25, n)
    k, v = np.zeros((rows, D), np.float16), np.zeros((rows, D), np.float16)
    k[:n, 0] = steps / 64  # scores of up to 3/8
    p = np.exp(steps / 64)
    first = (r.choice([-1, 1], (n // 2, D)) * r.uniform(0.25, 0.45, (n // 2, D))).astype(np.float16)
    v[:n:2], v[1:n:2] = first, (-first * (p[::2] / p[1::2])[:, None]).astype(np.float16)
    j = np.arange(rows)
    pool.K[pool.table[0, j // 16], 0, j % 16], pool.V[pool.table[0, j // 16], 0, j % 16] = k, v
    q = np.zeros((m, g, D), np.float16)
    q[:, :, 0] = 1
    got = pk.paged_attend(config(1, g), gpu(q), pool.cache(), ints(pool.table), ints([rows]), ints([0, m]), 1.0,
                          max_tokens=most).cpu().numpy()
    want = attend64(q, k, v, np.arange(n, rows), np.ones(rows, bool), 1.0, 0.0, None)
    # Of the largest value: 2^-20, twice the rounding of the scores' factor and products (2^-22 of 3/8), 2^-33 a row; and
    # the output's own.
    tol = (2.0 ** -20 + 2 * 2.0 ** -22 * 0.375 + rows * 2.0 ** -33) * np.abs(v.astype(np.float64)).max()
    tol = tol + np.abs(want) * 2.0 ** -11 + 2.0 ** -25
    off = np.abs(got.astype(np.float64) - want) / tol
    assert (off <= 1).all(), f"off by {off.max():.3g} of what is allowed"
