"""Values of V that are not finite, over long sequences and beside pages that are none."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
from new_tokens import D, SCALE, check, gpu
from pages import Pool, attend64, config, ints, tolerance

pytestmark = pytest.mark.gpu


def _fastest_us(call, runs=5):
    times = []
    for _ in range(runs):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        call()
        end.record()
        torch.cuda.synchronize()
        times.append(1000 * begin.elapsed_time(end))
    return min(times)


@pytest.mark.parametrize("m", [1, 8])
@pytest.mark.parametrize("lost", [(), (3,), (3, 7001)])
def test_the_keys_before_are_not_walked_once_more(m, lost):
    # A call looks at a step's 32 keys once more: 40 trips to memory of up to 2 us each.  Three such steps fit a
    # millisecond; a walk over all keys of the sequence would be 131067 trips.
    n, g, page, pages = 131067, 4, 16, 8192
    print(f"[paged] {m} tokens over {n} rows, lost pages {lost}", flush=True)
    cache = pk.PagedCache(*(torch.randn(pages, 1, page, D, device="cuda").half() for _ in range(2)))
    table = np.arange(pages)[None].copy()
    table[0, list(lost)] = -1
    table = ints(table)
    cfg = config(1, g)
    q = torch.randn(m, g, D, device="cuda").half()
    out = torch.zeros_like(q)
    ws = torch.empty(pk.paged_workspace_size(cfg, 1, m), dtype=torch.uint8, device="cuda")

    def call():
        pk.paged_attend(cfg, q, cache, table, ints_n, offsets, SCALE, out=out, workspace=ws)

    ints_n, offsets = ints([n]), ints([0, m])
    finite = _fastest_us(call)
    want = out.clone()
    assert torch.isfinite(want).all()
    cache.V[-1, 0, (n - 1) % page, 7] = float("inf")  # the last token's own row
    for j in lost:  # a row of the same step as those that are not there
        cache.V[j - 1, 0, 0, 9 + j % 64] = float("nan")
    odd = _fastest_us(call)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[-1, :, 7] = True
    for j in lost:
        hit[:, :, 9 + j % 64] = True
    assert not torch.isfinite(out[hit]).any() and torch.equal(out[~hit], want[~hit])
    assert odd < finite + 1000, f"{odd:.0f} us, {finite:.0f} without"


# Stretches of many steps a wave, and of several heads and sequences; the steps beside lost pages hold such values, and
# so do some that every token sees whole.
@pytest.mark.parametrize("batch,n,hkv,m,g,page", [(16, 5000, 8, 1, 4, 16), (16, 5000, 8, 4, 4, 16), (16, 5000, 8, 8, 4, 16),
                                                  (5, 900, 3, 3, 7, 7), (40, 130, 2, 2, 4, 100), (3, 20000, 1, 5, 5, 48)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_values_beside_lost_pages(batch, n, hkv, m, g, page, cap):
    print(f"[paged] not finite: {batch} x {n} hkv {hkv} m {m} g {g} page {page} cap {cap}", flush=True)
    r = np.random.default_rng(n + m)
    lens = [int(x) for x in r.integers(n // 2, n + 1, batch)]
    pool = Pool(r, hkv, lens, page)
    there, odd = [], []
    for b, rows in enumerate(lens):
        held = -(-rows // page)
        lost = np.unique(r.integers(0, held, max(1, held // 60))) if b % 3 else np.array([], np.int64)
        j = np.arange(rows)
        there.append(~np.isin(j // page, lost))
        places = [int(x) for x in np.concatenate((r.integers(0, rows, 3), lost * page - 1, lost * page + page, lost * page))
                  if 0 <= x < rows] + [rows - 1, rows - m]
        if b % 4 == 3:
            places = places[:3]
        v = pool.rows[b][1].astype(np.float32)
        for i, x in enumerate(places):
            v[x, :, (11 * i + b) % 100] = (np.inf, -np.inf, np.nan)[i % 3]
        pool.V[pool.table[b, j // page], :, j % page] = v
        odd.append(v)
        pool.table[b, lost] = [-1, len(pool.K), 2 ** 31 - 1][b % 3]
    q = r.standard_normal((batch * m, hkv * g, D)).astype(np.float16)
    got = pk.paged_attend(config(hkv, g), gpu(q), pool.cache(), ints(pool.table), ints(lens), ints(np.arange(batch + 1) * m),
                          SCALE, max_tokens=m, softcap=cap).cpu().numpy()
    for b in range(0, batch, 1 if batch < 10 else 3):
        p = np.arange(lens[b] - m, lens[b])
        for h in (0, hkv - 1):
            k, bad = pool.rows[b][0][:, h], odd[b][:, h]
            v = np.where(np.isfinite(bad), bad, 0)
            qh = q[b * m:(b + 1) * m].reshape(m, hkv, g, D)[:, h]
            want, tol = attend64(qh, k, v, p, there[b], SCALE, cap, None), tolerance(qh, k, v, SCALE, cap)
            x = got[b * m:(b + 1) * m].reshape(m, hkv, g, D)[:, h].astype(np.float32)
            for i in range(m):
                hit = ~np.isfinite(bad[:p[i] + 1][there[b][:p[i] + 1]]).all(0)
                assert not np.isfinite(x[i][:, hit]).any(), f"seq {b} head {h} token {i}"
                check(x[i][:, ~hit], want[i][:, ~hit], tol, f"seq {b} head {h} token {i}")


@pytest.mark.parametrize("m,g", [(1, 4), (4, 8)])
def test_rows_that_overflowed_in_keys_and_values(m, g):
    # A row of infinities in K and V: its score is infinite or NaN, its tokens' outputs are not finite in any dim where
    # the row's value is not; tokens before it are as without it.
    r = np.random.default_rng(m)
    for n in (40, 700, 30000):
        pool = Pool(r, 1, [n], 16)
        q = np.abs(r.standard_normal((m, g, D))).astype(np.float16)
        args = (config(1, g), gpu(q))
        rest = (ints(pool.table), ints([n]), ints([0, m]), SCALE)
        want = pk.paged_attend(*args, pool.cache(), *rest, max_tokens=m).cpu().numpy()
        for sign in (1, -1):
            pool.K[pool.table[0, (n - 1) // 16], 0, (n - 1) % 16] = sign * np.inf
            pool.V[pool.table[0, (n - 1) // 16], 0, (n - 1) % 16] = np.inf
            got = pk.paged_attend(*args, pool.cache(), *rest, max_tokens=m).cpu().numpy()
            assert not np.isfinite(got[-1]).any()
            tol = 2 * tolerance(q, pool.rows[0][0][:, 0], pool.rows[0][1][:, 0], SCALE)
            check(got[:-1], want[:-1].astype(np.float64), tol, f"{n} rows")
