"""GPU parity of the attention of packed new tokens over pages, against float64."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
from new_tokens import D, SCALE, check, gpu
from pages import Pool, attend64, config, ints, tolerance

pytestmark = pytest.mark.gpu


def _slopes(hq):
    return np.array([2.0 ** (-8 * (i + 1) / hq) for i in range(hq)], dtype=np.float32)


def _expect(pool, q, offsets, counts, hkv, g, scale, cap, slopes, got, heads=None, lost=()):
    """Every output of every sequence against float64; lost: pages that tables name but that are none."""
    for b, n in enumerate(pool.lens):
        m = counts[b]
        if m == 0:
            continue
        rows = slice(offsets[b], offsets[b] + m)
        k, v = pool.rows[b]
        there = ~np.isin(np.arange(n) // pool.page, [j for s, j in lost if s == b])
        positions = np.arange(n - m, n)
        for h in (range(hkv) if heads is None else heads):
            qh = q[rows].reshape(m, hkv, g, D)[:, h]
            sl = None if slopes is None else slopes[h * g:(h + 1) * g]
            want = attend64(qh, k[:, h], v[:, h], positions, there, scale, cap, sl)
            tol = tolerance(qh, k[:, h], v[:, h], scale, cap, sl)
            check(got[rows].reshape(m, hkv, g, D)[:, h], want, tol, f"seq {b} head {h}")


def _run(lens, counts, hkv, g, page, scale=SCALE, cap=0.0, bias=False, law=1.0, most=None, pad=2, some=None, seed=0,
         heads=None, lost=(), q_wide=False):
    """One call checked in every output.  Rows that no sequence has hold NaN, as do the queries of padding; rows of out that
    no sequence has have to stay as they were.  some: the counts that are passed beside the offsets."""
    print(f"[paged] batch {len(lens)} lens {lens[:8]} counts {counts[:8]} hkv {hkv} g {g} page {page} cap {cap} bias {bias} "
          f"most {most}", flush=True)
    r = np.random.default_rng(seed)
    hq = hkv * g
    pool = Pool(r, hkv, lens, page, law)
    for b, j in lost:
        pool.table[b, j] = [-1, len(pool.K), 2 ** 31 - 1, -2 ** 31][(b + j) % 4]
    offsets = np.concatenate(([0], np.cumsum(counts)))
    t = int(offsets[-1]) + pad
    q = (law * r.standard_normal((t, hq, D))).astype(np.float16)
    real = list(counts) if some is None else [min(max(x, 0), y) for x, y in zip(some, counts)]
    kept = np.ones(t, dtype=bool)
    for b, m in enumerate(real):
        kept[offsets[b]:offsets[b] + m] = False
    q[kept] = np.nan
    slopes = _slopes(hq) if bias else None
    out = torch.full((t, hq, D), 7.0, dtype=torch.float16, device="cuda")
    gq = gpu(q)
    if q_wide:  # the first columns of a wider product
        gq = torch.cat((gq, torch.full((t, 3, D), 5.0, dtype=torch.float16, device="cuda")), 1)[:, :hq]
    got = pk.paged_attend(config(hkv, g), gq, pool.cache(), ints(pool.table), ints(lens), ints(offsets), scale,
                          counts=None if some is None else ints(some), max_tokens=max(max(counts), 1) if most is None else most,
                          softcap=cap, slopes=None if slopes is None else gpu(slopes), out=out).cpu().numpy()
    assert (got[kept] == 7).all(), "rows of tokens that no sequence has were written"
    # With fewer tokens than the offsets say, the last one still stands at lens - 1.
    _expect(pool, q, offsets, real, hkv, g, scale, cap, slopes, got, heads, lost)
    return got


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 5000])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 100])
def test_single_tokens(n, page):
    _run([n], [1], 2, 4, page, seed=n)


@pytest.mark.parametrize("g", [1, 2, 3, 4, 5, 7, 8, 11, 16])
@pytest.mark.parametrize("m", [1, 2, 3, 9])
def test_heads_per_kv_head(g, m):
    _run([300, m, 77 + m], [m, m, 1], 3, g, 16, seed=g)


@pytest.mark.parametrize("batch", [2, 64, 255, 256, 257, 700])
def test_wide_batches(batch):
    r = np.random.default_rng(batch)
    lens = [int(x) for x in r.integers(1, 200, batch)]
    _run(lens, [1] * batch, 1, 4, 16, seed=batch)
    counts = [int(min(x, y)) for x, y in zip(r.integers(0, 12, batch), lens)]
    _run(lens, counts, 1, 4, 16, seed=batch, most=12)


@pytest.mark.parametrize("page", [16, 48, 512])
def test_lengths_far_apart(page):
    # Blocks share the long ones' keys and take several of the short ones.
    r = np.random.default_rng(page)
    lens = [40000, 1, 2, 9000, 128, 129, 20000] + [int(x) for x in r.integers(1, 60, 30)]
    _run(lens, [1] * len(lens), 2, 4, page, seed=1)
    _run(lens, [min(n, 2) for n in lens], 2, 8, page, seed=2)
    _run(lens, [min(n, 30) for n in lens], 2, 4, page, seed=3)


def test_sequences_without_tokens_and_without_rows():
    _run([50, 0, 7, 300, 0], [0, 0, 7, 1, 0], 2, 2, 16)
    _run([50, 0, 70, 300, 0], [0, 0, 70, 1, 0], 2, 2, 16)
    _run([0, 0, 0], [0, 0, 0], 2, 2, 16)
    _run([0, 0, 0], [0, 0, 0], 2, 2, 16, most=40)


@pytest.mark.parametrize("batch,step", [(40, 7), (300, 64), (300, 65), (1000, 333)])
def test_batches_of_mostly_empty_places(batch, step):
    # Every step-th place has a sequence; of those between some have rows, but no new tokens.
    lens = [3 * (b % 5) for b in range(batch)]
    for m in (1, 40):
        counts = [0] * batch
        for b in range(step // 2, batch, step):
            lens[b], counts[b] = 700 + b, m
        _run(lens, counts, 2, 2, 16, seed=m)
        counts[step // 2] = 1
        _run(lens, counts, 2, 2, 16, seed=m, most=40)


@pytest.mark.parametrize("most", [4, 100])
def test_tokens_that_attend_nothing_give_zeros(most):
    # No row at all, and more tokens than rows: those at positions below 0 see nothing.
    hkv, g = 2, 3
    r = np.random.default_rng(1)
    pool = Pool(r, hkv, [0, 2, 5], 16)
    q = r.standard_normal((9, hkv * g, D)).astype(np.float16)
    got = pk.paged_attend(config(hkv, g), gpu(q), pool.cache(), ints(pool.table), ints([0, 2, 5]), ints([0, 2, 6, 9]), SCALE,
                          max_tokens=most).cpu().numpy()
    assert (got[:4] == 0).all()
    for b, m, lo in ((1, 2, 4), (2, 3, 6)):
        for h in range(hkv):
            k, v = (x[:, h] for x in pool.rows[b])
            qh = q[lo:lo + m].reshape(m, hkv, g, D)[:, h]
            n = pool.lens[b]
            want = attend64(qh, k, v, np.arange(n - m, n), np.ones(n, bool), SCALE, 0.0, None)
            check(got[lo:lo + m].reshape(m, hkv, g, D)[:, h], want, tolerance(qh, k, v, SCALE), f"seq {b}")


@pytest.mark.parametrize("m", [1, 5, 100])
def test_fewer_tokens_than_offsets_say(m):
    _run([300, 200, 150, 400, 500], [m] * 5, 2, 4, 16, some=[m, 0, -3, m + 9, max(1, m // 2)], seed=m)


def test_tokens_past_max_tokens_are_not_computed():
    for m, most in ((9, 4), (300, 50)):
        _run([400, 500], [m, 3], 2, 4, 16, some=[most, 3], most=most, seed=m)
        r = np.random.default_rng(3)
        pool = Pool(r, 2, [400, 500], 16)
        q = r.standard_normal((m + 3, 8, D)).astype(np.float16)
        args = (config(2, 4), gpu(q), pool.cache(), ints(pool.table), ints(pool.lens), ints([0, m, m + 3]), SCALE)
        a = pk.paged_attend(*args, max_tokens=most, out=torch.full((m + 3, 8, D), 7.0, dtype=torch.float16, device="cuda"))
        b = pk.paged_attend(*args, max_tokens=most, counts=ints([most, 3]), out=torch.full_like(a, 7.0))
        assert torch.equal(a, b) and (a[most:m] == 7).all()


@pytest.mark.parametrize("t", [33, 63, 64, 65, 127, 128, 129, 257, 500])
@pytest.mark.parametrize("page", [16, 48])
def test_prompts(t, page):
    _run([t], [t], 2, 2, page, seed=t)
    _run([t + 700, t, 901], [t, t, 1], 1, 3, page, seed=t)


@pytest.mark.parametrize("g", [1, 3, 4, 7, 16])
@pytest.mark.parametrize("page", [1, 7, 100, 4096])
def test_chunks(g, page):
    _run([1000, 333], [140, 1], 2, g, page, seed=g)


@pytest.mark.parametrize("hkv", [1, 8])
def test_chunks_among_single_tokens(hkv):
    # Few tiles of rows and long lengths: keys are cut into shares; short sequences stay whole.
    r = np.random.default_rng(hkv)
    lens = [9000, 64, 30000, 1, 700] + [int(x) for x in r.integers(1, 3000, 20)]
    counts = [200, 1, 1, 1, 65] + [1] * 20
    _run(lens, counts, hkv, 4, 32, seed=1, heads=[0, hkv - 1])


def test_wide_batches_of_chunks():
    r = np.random.default_rng(3)
    lens = [int(x) for x in r.integers(1, 400, 300)]
    counts = [int(min(x, y)) for x, y in zip(r.integers(0, 60, 300), lens)]
    _run(lens, counts, 2, 2, 16, seed=4)


# Tiles of rows whose keys several blocks share: few of them, over many keys.
@pytest.mark.parametrize("lens,counts,hkv,g", [([6000], [40], 2, 4), ([5000, 30, 7001], [64, 1, 33], 1, 3),
                                               ([3000, 2500, 2000], [300, 290, 1], 2, 2), ([12000], [130], 1, 16)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_tiles_that_blocks_share(lens, counts, hkv, g, cap, bias):
    _run(lens, counts, hkv, g, 16, cap=cap, bias=bias, seed=len(lens))
    lost = [(b, j) for b, n in enumerate(lens) for j in ([0, 3] + list(range(n // 32, n // 32 + 9)) if n > 1000 else [])]
    _run(lens, counts, hkv, g, 16, cap=cap, bias=bias, lost=lost, seed=7)


@pytest.mark.parametrize("lens,counts", [([8000], [1200]), ([9000, 6000], [300, 700])])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_tiles_that_few_blocks_share(lens, counts, cap):
    _run(lens, counts, 2, 4, 16, cap=cap, seed=9, heads=[1], lost=[(0, j) for j in range(40, 60)])


@pytest.mark.parametrize("n,m,hkv,g", [(30000, 1, 1, 4), (30000, 4, 1, 8), (70000, 20, 1, 4), (33000, 3, 2, 16)])
def test_one_long_sequence(n, m, hkv, g):
    # All blocks share the keys of a head or two.
    _run([n], [m], hkv, g, 16, seed=m)
    _run([n], [m], hkv, g, 16, seed=m, lost=[(0, j) for j in range(200, 900)])


def test_tiles_that_blocks_share_in_wide_batches():
    # Several sequences a lane, of which few are long.
    r = np.random.default_rng(5)
    lens = [int(x) for x in r.integers(1, 300, 200)]
    counts = [int(min(x, y)) for x, y in zip(r.integers(0, 40, 200), lens)]
    for b in (0, 1, 77, 199):
        lens[b], counts[b] = 9000 + b, 35
    _run(lens, counts, 1, 2, 16, seed=6)


# More tiles of rows than blocks that the chip holds at once: the last round of them full, or not, or begun by another
# sequence (of equal tiles or not).
@pytest.mark.parametrize("lens,counts,hkv", [([2048], [2048], 8), ([2100], [2100], 8), ([1500, 1200], [1500, 1200], 8),
                                             ([3000], [2100], 8), ([700, 2000, 900], [600, 1100, 450], 8)])
def test_many_tiles(lens, counts, hkv):
    _run(lens, counts, hkv, 4, 64, seed=3, heads=[0, hkv - 1])


@pytest.mark.parametrize("cap,bias", [(20.0, False), (1.0, False), (0.0, True), (30.0, True), (1e4, False)])
@pytest.mark.parametrize("lens,counts,g", [([500, 33], [1, 1], 4), ([500, 33], [9, 2], 3), ([700, 90], [150, 1], 4)])
def test_shaped_scores(cap, bias, lens, counts, g):
    _run(lens, counts, 2, g, 16, cap=cap, bias=bias, seed=2)
    _run(lens, counts, 2, g, 16, cap=cap, bias=bias, law=4.0, seed=3)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.4])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (5.0, False), (0.0, True)])
def test_scales(scale, cap, bias):
    _run([200, 60], [1, 1], 2, 2, 16, scale=scale, cap=cap, bias=bias)
    _run([200, 60], [70, 1], 2, 2, 16, scale=scale, cap=cap, bias=bias)


def test_steep_biases():
    # Slopes whose bias at the far end is beyond every exponential.
    r = np.random.default_rng(8)
    for n, m in ((20000, 1), (20000, 40)):
        pool = Pool(r, 1, [n], 16)
        q = r.standard_normal((m, 2, D)).astype(np.float16)
        slopes = np.array([100.0, -0.01], dtype=np.float32)
        got = pk.paged_attend(config(1, 2), gpu(q), pool.cache(), ints(pool.table), ints([n]), ints([0, m]), SCALE,
                              max_tokens=m, slopes=gpu(slopes)).cpu().numpy()
        k, v = (x[:, 0] for x in pool.rows[0])
        want = attend64(q, k, v, np.arange(n - m, n), np.ones(n, bool), SCALE, 0.0, slopes)
        # The second head's bias grows to 200: its rounding is that of scores as large.
        tol = tolerance(q, k, v, SCALE, 0.0, slopes) + 2 * 2.0 ** -23 * 200 * np.abs(v.astype(np.float64)).max()
        check(got, want, tol, f"{m} tokens")


@pytest.mark.parametrize("lens,counts,lost", [
    ([100], [1], [(0, 2)]), ([300, 40], [1, 1], [(0, 0), (0, 18), (1, 2)]), ([64], [1], [(0, 0), (0, 1), (0, 2), (0, 3)]),
    ([500, 200], [90, 1], [(0, 0), (0, 5), (0, 31), (1, 12)]), ([200], [200], [(0, j) for j in range(4)]),
    ([3000], [4], [(0, j) for j in range(100, 180)])])
@pytest.mark.parametrize("cap", [0.0, 10.0])
def test_rows_of_pages_that_are_none_are_attended_by_nobody(lens, counts, lost, cap):
    _run(lens, counts, 2, 4, 16, lost=lost, cap=cap, seed=5)


@pytest.mark.parametrize("lens,counts,g,page", [
    ([500], [1], 4, 16), ([500, 90], [5, 1], 3, 7), ([4000, 90], [8, 1], 4, 16), ([600, 300], [100, 40], 2, 16),
    ([9000], [70], 4, 64), ([300], [300], 2, 48)])
def test_rows_that_are_not_finite_reach_only_tokens_that_see_them(lens, counts, g, page):
    print(f"[paged] not finite: lens {lens} counts {counts} g {g} page {page}", flush=True)
    hkv = 2
    r = np.random.default_rng(sum(lens))
    pool = Pool(r, hkv, lens, page)
    offsets = np.concatenate(([0], np.cumsum(counts)))
    q = r.standard_normal((int(offsets[-1]), hkv * g, D)).astype(np.float16)
    odds = []
    for b, (n, m) in enumerate(zip(lens, counts)):
        # The last token's own row, one among the new tokens, one before them, and a key that makes scores NaN.
        values = {n - 1: np.inf, n - 1 - m // 2: np.nan, (n - m) // 2: -np.inf}
        lost = n - m + m // 3 if m > 2 else -1
        for j in values:
            at = pool.table[b, j // page]
            for i, x in enumerate(values.values()):
                if list(values)[i] == j:
                    pool.V[at, :, j % page, 5 + 30 * i] = pool.V[at, :, j % page, 127] = x
        if lost >= 0:
            pool.K[pool.table[b, lost // page], :, lost % page, 77] = np.nan
        odds.append(lost)
    got = pk.paged_attend(config(hkv, g), gpu(q), pool.cache(), ints(pool.table), ints(lens), ints(offsets), SCALE,
                          max_tokens=max(counts)).cpu().numpy()
    for b, (n, m) in enumerate(zip(lens, counts)):
        j = np.arange(n)
        at = pool.table[b, j // page]
        p = np.arange(n - m, n)
        for h in range(hkv):
            bad = pool.V[at, h, j % page].astype(np.float32)
            v = np.where(np.isfinite(bad), bad, 0)
            k = np.where(np.isfinite(pool.K[at, h, j % page]), pool.K[at, h, j % page], 0)
            x = got[offsets[b]:offsets[b + 1]].reshape(m, hkv, g, D)[:, h].astype(np.float32)
            dead = p >= odds[b] if odds[b] >= 0 else np.zeros(m, bool)
            assert np.isnan(x[dead]).all()
            qh = q[offsets[b]:offsets[b + 1]].reshape(m, hkv, g, D)[:, h]
            want = attend64(qh, k, v, p, np.ones(n, bool), SCALE, 0.0, None)
            tol = tolerance(qh, k, v, SCALE)
            for i in range(m):
                if dead[i]:
                    continue
                hit = ~np.isfinite(bad[:p[i] + 1]).all(0)
                assert not np.isfinite(x[i][:, hit]).any()
                check(x[i][:, ~hit], want[i][:, ~hit], tol, f"seq {b} head {h} token {i}")


def test_queries_that_are_not_finite_make_their_own_outputs_nan():
    r = np.random.default_rng(2)
    for m in (3, 60):
        pool = Pool(r, 1, [200], 16)
        q = r.standard_normal((m, 4, D)).astype(np.float16)
        q[1, 2, 7] = np.nan
        got = pk.paged_attend(config(1, 4), gpu(q), pool.cache(), ints(pool.table), ints([200]), ints([0, m]), SCALE,
                              max_tokens=m).cpu().numpy()
        assert np.isnan(got[1, 2]).all()
        got[1, 2] = 0
        assert np.isfinite(got).all()


@pytest.mark.parametrize("m", [1, 3, 50])
@pytest.mark.parametrize("shift", [3000.0, -60000.0])
def test_large_scores_are_weighed_by_their_differences(m, shift):
    # Scores near `shift` 4, exact in float32: their first dim is common to all keys, the others small.
    r = np.random.default_rng(6)
    n, g = 700, 2
    pool = Pool(r, 1, [n], 16)
    j = np.arange(n)
    k = (r.integers(-8, 9, (n, D)) / 4).astype(np.float16)
    k[:, 0] = 4.0
    pool.K[pool.table[0, j // 16], 0, j % 16] = k
    q = (r.integers(-4, 5, (m, g, D)) / 4).astype(np.float16)
    q[:, :, 0] = shift
    got = pk.paged_attend(config(1, g), gpu(q), pool.cache(), ints(pool.table), ints([n]), ints([0, m]), 0.25,
                          max_tokens=m).cpu().numpy()
    v = pool.rows[0][1][:, 0]
    want = attend64(q, k, v, np.arange(n - m, n), np.ones(n, bool), 0.25, 0.0, None)
    # Products and sums are multiples of 1/16 below 2^18 + 2^10: exact in float32.  What is left of a score's rounding is
    # that of the differences (below 2^9).
    tol = (2 * (2.0 ** -22 * 2 ** 9 + 2.0 ** -20) + 2.0 ** -10) * np.abs(v.astype(np.float64)).max()
    check(got, want, tol, f"{m} tokens")


def test_strided_queries_and_defaults():
    _run([300, 77], [1, 1], 2, 4, 16, q_wide=True)
    _run([300, 177], [1, 90], 2, 4, 16, q_wide=True)
    r = np.random.default_rng(1)
    pool = Pool(r, 2, [50, 60], 16)
    q = gpu(r.standard_normal((4, 8, D)).astype(np.float16))
    args = (config(2, 4), q, pool.cache(), ints(pool.table), ints([50, 60]), ints([0, 1, 4]), SCALE)
    a, b = pk.paged_attend(*args), pk.paged_attend(*args, max_tokens=3)
    assert a.shape == (4, 8, D) and a.dtype == torch.float16 and torch.equal(a, b)


def test_a_dense_cache_is_one_of_pages():
    r = np.random.default_rng(4)
    b, hkv, g, n = 3, 2, 4, 777
    K, V = (r.standard_normal((b, hkv, n, D)).astype(np.float16) for _ in range(2))
    q = r.standard_normal((b, hkv * g, D)).astype(np.float16)
    cfg = config(hkv, g)
    got = pk.paged_attend(cfg, gpu(q), pk.PagedCache(gpu(K), gpu(V)), ints(np.arange(b)[:, None]), ints([n] * b),
                          ints(np.arange(b + 1)), SCALE, max_tokens=1)
    dense = pk.sink_window_attend(cfg, gpu(q[:, :, None]), gpu(K), gpu(V), n - 1, 0, n, SCALE)[:, :, 0]
    for h in range(hkv * g):
        for s in range(b):
            tol = tolerance(q[s, h], K[s, h // g], V[s, h // g], SCALE)
            check(got[s, h].cpu().numpy(), dense[s, h].double().cpu().numpy(), 2 * tol, f"seq {s} head {h}")


def test_sequences_that_share_pages():
    r = np.random.default_rng(4)
    pool = Pool(r, 2, [320], 16)
    table = np.concatenate((pool.table, pool.table, pool.table))
    q = np.repeat(r.standard_normal((1, 4, D)).astype(np.float16), 3, 0)
    got = pk.paged_attend(config(2, 2), gpu(q), pool.cache(), ints(table), ints([320, 320, 320]), ints([0, 1, 2, 3]), SCALE,
                          max_tokens=1)
    for i in (1, 2):  # blocks cut the three in different places
        tol = max(tolerance(q[0], pool.rows[0][0][:, h], pool.rows[0][1][:, h], SCALE) for h in range(2))
        check(got[i].cpu().numpy(), got[0].double().cpu().numpy(), 2 * tol, f"copy {i}")


@pytest.mark.parametrize("most", [2, 40])
def test_values_out_of_range_stay_in_bounds(most):
    big, low = 2 ** 31 - 1, -2 ** 31
    r = np.random.default_rng(3)
    pool = Pool(r, 1, [100, 100, 100], 16)
    q = gpu(r.standard_normal((50, 2, D)).astype(np.float16))
    cache, table = pk.PagedCache(*(torch.nan_to_num(x) for x in (pool.cache().K, pool.cache().V))), ints(pool.table)
    for lens, offsets, counts in (([big, low, 100], [0, 3, 5, 6], None), ([100] * 3, [low, big, 7, big], None),
                                  ([100] * 3, [0, 50, 0, 50], None), ([5, 100, 100], [0, 20, 40, 60], [big, low, 3]),
                                  ([100] * 3, [40, 30, 20, 10], [7, 7, 7])):
        pk.paged_attend(config(1, 2), q, cache, table, ints(lens), ints(offsets), SCALE,
                        counts=None if counts is None else ints(counts), max_tokens=most)
        torch.cuda.synchronize()


@pytest.mark.parametrize("most", [1, 8, 64])
def test_captured_calls_replay_with_other_lengths(most):
    r = np.random.default_rng(most)
    hkv, g, batch, page, width = 2, 4, 20, 16, 130
    t = batch * most
    pages = batch * width
    cache = pk.PagedCache(*(torch.randn(pages, hkv, page, D, device="cuda").half() for _ in range(2)))
    table, lens, offsets = ints(np.zeros((batch, width))), ints(np.ones(batch)), ints(np.arange(batch + 1))
    cfg = config(hkv, g)
    q = torch.randn(t, hkv * g, D, device="cuda").half()
    ws = torch.empty(pk.paged_workspace_size(cfg, batch, t, most), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(2)]

    def call(out):
        pk.paged_attend(cfg, q, cache, table, lens, offsets, SCALE, max_tokens=most, out=out, workspace=ws)

    call(outs[0])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]  # two graphs that share a workspace
    for graph, out in zip(graphs, outs):
        with torch.cuda.graph(graph):
            call(out)
    for i in range(4):
        n = np.maximum(r.integers(1, width * page + 1, batch), most)
        n[: i] = most
        lens.copy_(ints(n))
        table.copy_(ints(r.permutation(pages).reshape(batch, width)))
        offsets.copy_(ints(np.concatenate(([0], np.cumsum(r.integers(0, most + 1, batch))))))
        q.normal_()
        for out in outs:
            out.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(q)
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_one_workspace_serves_smaller_calls():
    cfg, r = config(2, 4), np.random.default_rng(1)
    pool = Pool(r, 2, [3000, 500, 70, 5000], 16)
    cache, table = pool.cache(), ints(pool.table)
    ws = torch.empty(pk.paged_workspace_size(cfg, 4, 400, 200), dtype=torch.uint8, device="cuda")
    for batch, m in ((4, 100), (4, 8), (4, 9), (3, 4), (2, 5), (1, 1), (2, 200)):
        assert pk.paged_workspace_size(cfg, batch, batch * m, m) <= ws.numel()
        q = gpu(r.standard_normal((batch * m, 8, D)).astype(np.float16))
        x, y = (pk.paged_attend(cfg, q, cache, table[:batch], ints(pool.lens[:batch]), ints(np.arange(batch + 1) * m), SCALE,
                                max_tokens=m, workspace=w, out=torch.zeros_like(q)) for w in (ws, None))
        assert torch.equal(x, y)


def test_calls_on_two_streams():
    cfg, r = config(2, 4), np.random.default_rng(1)
    pool = Pool(r, 2, [20000, 500, 70, 5000], 16)
    cache, table, lens = pool.cache(), ints(pool.table), ints(pool.lens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for m in (1, 60):
        qs = [gpu(r.standard_normal((4 * m, 8, D)).astype(np.float16)) for _ in range(2)]
        offsets = ints(np.arange(5) * m)
        want = [pk.paged_attend(cfg, q, cache, table, lens, offsets, SCALE, max_tokens=m) for q in qs]
        torch.cuda.synchronize()
        got = [pk.paged_attend(cfg, q, cache, table, lens, offsets, SCALE, max_tokens=m, stream=s) for q, s in zip(qs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_pages_past_four_gigabytes():
    # 9.2 GB of keys and as much of values; the sequences' pages lie in their last part.
    r = np.random.default_rng(11)
    hkv, g, page, pages = 8, 2, 64, 70000
    cfg = config(hkv, g)
    cache = pk.PagedCache.empty(cfg, pages, page)
    lens, counts = [700, 100], [1, 40]
    held = [11, 2]
    mine = pages - 1 - r.permutation(3000)[:13]
    table = np.full((2, 12), -1)
    table[0, :11], table[1, :2] = mine[:11], mine[11:]
    rows = []
    for b, n in enumerate(lens):
        x = r.standard_normal((n, hkv * g + 2 * hkv, D)).astype(np.float16)
        j = np.arange(n)
        gx = gpu(x)
        pk.rotate_rows(cfg, cache, gx[:, :16], gx[:, 16:24], gx[:, 24:], ints(j), ints(table[b, j // page] * page + j % page))
        rows.append((x[:, 16:24], x[:, 24:]))
        at = gpu(table[b, j // page].astype(np.int64))
        assert torch.equal(cache.K[at, :, gpu(j % page)], gx[:, 16:24]) and torch.equal(cache.V[at, :, gpu(j % page)], gx[:, 24:])
    for most in (1, 40):
        m = [min(c, most) for c in counts]
        q = r.standard_normal((sum(m), hkv * g, D)).astype(np.float16)
        got = pk.paged_attend(cfg, gpu(q), cache, ints(table), ints(lens), ints([0, m[0], sum(m)]), SCALE,
                              max_tokens=most).cpu().numpy()
        for b, n in enumerate(lens):
            lo = 0 if b == 0 else m[0]
            for h in range(hkv):
                k, v = (x[:, h] for x in rows[b])
                qh = q[lo:lo + m[b]].reshape(m[b], hkv, g, D)[:, h]
                want = attend64(qh, k, v, np.arange(n - m[b], n), np.ones(n, bool), SCALE, 0.0, None)
                check(got[lo:lo + m[b]].reshape(m[b], hkv, g, D)[:, h], want, tolerance(qh, k, v, SCALE), f"seq {b} head {h}")


@pytest.mark.parametrize("most", [1, 40])
def test_the_widest_batch(most):
    # 65535 sequences of one row, whose output is its value, and some longer ones among them.
    r = np.random.default_rng(12)
    batch, long = 65535, {5: 300, 40000: 70, 65534: 129}
    cache = pk.PagedCache(*(torch.randn(batch + 50, 1, 16, D, device="cuda").half() for _ in range(2)))
    table, lens = np.zeros((batch, 19), np.int64), np.ones(batch, np.int64)
    perm = r.permutation(batch + 50)
    table[:, 0] = perm[:batch]
    for b, n in long.items():
        lens[b] = n
        table[b, 1:] = r.integers(0, batch + 50, 18)
    q = torch.randn(batch, 2, D, device="cuda").half()
    got = pk.paged_attend(config(1, 2), q, cache, ints(table), ints(lens), ints(np.arange(batch + 1)), SCALE, max_tokens=most)
    one = torch.from_numpy(lens == 1).cuda()
    v = cache.V[torch.from_numpy(table[:, 0]).cuda(), 0, 0]
    assert torch.equal(got[one], v[one][:, None].expand(-1, 2, -1))
    for b, n in long.items():
        j = np.arange(n)
        k_, v_ = (x[torch.from_numpy(table[b, j // 16]).cuda(), 0, torch.from_numpy(j % 16).cuda()].cpu().numpy()
                  for x in (cache.K, cache.V))
        qb = q[b].cpu().numpy()[None]
        want = attend64(qb, k_, v_, [n - 1], np.ones(n, bool), SCALE, 0.0, None)
        check(got[b][None].cpu().numpy(), want, tolerance(qb, k_, v_, SCALE), f"seq {b}")
