"""Rows on their way into a paged cache against the same in 64 bits."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
from pages import config, ints, rotate64
from new_tokens import D, gpu

pytestmark = pytest.mark.gpu

EPS = 1e-6


def _freqs(rot, base=10000.0):
    return None if rot == 0 else np.array([base ** (-2 * i / rot) for i in range(rot // 2)], dtype=np.float32)


def _close(got, want, pair, what):
    """An output within half a float16 step (2^-11 of it, 2^-25 below float16's normal numbers) and what float32 leaves of
    the pair's length L: sine and cosine are off by 2^-22 (the angle's and their own rounding), the norm by 2^-21 (128
    squares summed, a root and three products), products and the sum by 2^-22, together under 2^-19."""
    got = np.asarray(got, dtype=np.float64)
    tol = np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + pair * 2.0 ** -19
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all(), f"{what}: off by {(np.abs(got - want) / tol).max():.3g} of what is allowed"


def _pair_length(y, rot, pairs):
    """The length of each value's pair (of itself where it is not rotated)."""
    n = np.abs(y)
    if rot:
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
        n[..., a] = n[..., b] = np.hypot(y[..., a], y[..., b])
    return n


def _run(t, hkv, g, page, rot=D, norm=True, pairs=False, layout="columns", far=100000, base=10000.0, law=1.0, seed=0):
    print(f"[rows] t {t} hkv {hkv} g {g} page {page} rot {rot} norm {norm} pairs {pairs} layout {layout}", flush=True)
    r = np.random.default_rng(seed)
    hq = hkv * g
    x = (law * r.standard_normal((t, hq + 2 * hkv, D))).astype(np.float16)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if layout == "columns":
        gx = gpu(x)
        gq, gk, gv = gx[:, :hq], gx[:, hq:hq + hkv], gx[:, hq + hkv:]
    else:
        gq, gk, gv = gpu(q), gpu(k), gpu(v)
    pages = -(-t // page) + 2
    slots = r.permutation(pages * page)[:t]
    slots[r.random(t) < 0.1] = -1
    if t > 3:
        slots[1], slots[2] = pages * page, 2 ** 31 - 1
    positions = r.integers(0, far, t)
    freqs = _freqs(rot, base)
    weights = [(1 + 0.2 * r.standard_normal(D)).astype(np.float32) if norm else None for _ in range(2)]
    K, V = (np.full((pages, hkv, page, D), 3.0, dtype=np.float16) for _ in range(2))
    cache = pk.PagedCache(gpu(K), gpu(V))
    q_out = gq if layout == "in place" else torch.full((t, hq, D), 7.0, dtype=torch.float16, device="cuda")
    pk.rotate_rows(config(hkv, g), cache, gq, gk, gv, ints(positions), ints(slots), None if freqs is None else gpu(freqs),
                   *(None if w is None else gpu(w) for w in weights), eps=EPS, pairs=pairs, q_out=q_out)
    out, gK, gV = (y.cpu().numpy() for y in (q_out, cache.K, cache.V))
    real = (slots >= 0) & (slots < pages * page)
    wq, wk = (rotate64(y, positions, freqs, w, EPS, pairs) for y, w in ((q, weights[0]), (k, weights[1])))
    untouched = q if layout == "in place" else np.full_like(q, 7.0)
    assert np.array_equal(out[~real], untouched[~real])
    _close(out[real], wq[real], _pair_length(wq, rot, pairs)[real], "q")
    at = slots[real]
    _close(gK[at // page, :, at % page], wk[real], _pair_length(wk, rot, pairs)[real], "k")
    assert np.array_equal(gV[at // page, :, at % page], v[real])
    # Every other row of the pages is left as it was.
    for y in (gK, gV):
        flat = y.transpose(0, 2, 1, 3).reshape(pages * page, hkv, D).copy()
        flat[at] = 3.0
        assert (flat == 3.0).all()


@pytest.mark.parametrize("t", [1, 2, 3, 17, 300, 2047, 2048, 2051])
@pytest.mark.parametrize("hkv,g,page", [(1, 1, 16), (8, 4, 64), (3, 5, 7), (2, 16, 1)])
def test_rows(t, hkv, g, page):
    _run(t, hkv, g, page, seed=t)


@pytest.mark.parametrize("rot", [0, 16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("t", [9, 2100])
def test_rotations(rot, pairs, norm, t):
    _run(t, 2, 3, 48, rot=rot, pairs=pairs, norm=norm, seed=rot)


@pytest.mark.parametrize("layout", ["columns", "apart", "in place"])
@pytest.mark.parametrize("t", [1, 5, 2500])
def test_layouts(layout, t):
    _run(t, 2, 4, 16, layout=layout, seed=t)


@pytest.mark.parametrize("far,base", [(2 ** 31 - 1, 10000.0), (4000000, 500000.0), (1, 10000.0), (2 ** 24 + 3, 1.0)])
def test_far_positions(far, base):
    _run(400, 1, 2, 16, far=far, base=base, seed=3)


def test_negative_positions_turn_back():
    r = np.random.default_rng(4)
    k = r.standard_normal((40, 1, D)).astype(np.float16)
    positions = r.integers(-1000000, 0, 40)
    cache = pk.PagedCache(*(torch.zeros(4, 1, 16, D, dtype=torch.float16, device="cuda") for _ in range(2)))
    out = pk.rotate_rows(config(1, 1), cache, gpu(k), gpu(k), gpu(k), ints(positions), ints(np.arange(40)),
                         gpu(_freqs(D))).cpu().numpy()
    want = rotate64(k, positions, _freqs(D), None, EPS, False)
    _close(out, want, _pair_length(want, D, False), "q")


@pytest.mark.parametrize("law", [1e-3, 30.0, 2000.0])
def test_small_and_large_rows(law):
    # Squares of 2000 pass float16's range, squares of 1e-3 fall below it; with eps they count less.
    _run(60, 2, 2, 16, law=law, seed=1)


def test_only_one_of_the_norms():
    r = np.random.default_rng(6)
    x = r.standard_normal((30, 2, D)).astype(np.float16)
    w = (1 + 0.2 * r.standard_normal(D)).astype(np.float32)
    for qw, kw in ((w, None), (None, w)):
        cache = pk.PagedCache(*(torch.zeros(2, 2, 16, D, dtype=torch.float16, device="cuda") for _ in range(2)))
        out = pk.rotate_rows(config(2, 1), cache, gpu(x), gpu(x), gpu(x), ints(np.arange(30)), ints(np.arange(30)),
                             q_weight=None if qw is None else gpu(qw), k_weight=None if kw is None else gpu(kw))
        got = cache.K.cpu().numpy().transpose(0, 2, 1, 3).reshape(32, 2, D)[:30]
        for y, v in ((out.cpu().numpy(), qw), (got, kw)):
            want = rotate64(x, None, None, v, EPS, False)
            _close(y, want, np.abs(want), "one norm")


def test_rows_of_zeros_and_rows_that_are_not_finite():
    x = np.zeros((3, 1, D), dtype=np.float16)
    x[1, 0, 5], x[2, 0, 100] = np.inf, np.nan
    w = np.ones(D, dtype=np.float32)
    cache = pk.PagedCache(*(torch.zeros(1, 1, 16, D, dtype=torch.float16, device="cuda") for _ in range(2)))
    out = pk.rotate_rows(config(1, 1), cache, gpu(x), gpu(x), gpu(x), ints([3, 4, 5]), ints([0, 1, 2]), gpu(_freqs(D)),
                         gpu(w), gpu(w)).cpu().numpy()
    assert (out[0] == 0).all() and np.isnan(out[1]).any() and np.isnan(out[2]).all()
    assert np.array_equal(cache.V[0, 0, :3].cpu().numpy(), x[:, 0], equal_nan=True)


def test_captured_calls_replay():
    r = np.random.default_rng(7)
    for t in (6, 2200):
        x = gpu(r.standard_normal((t, 4, D)).astype(np.float16))
        cache = pk.PagedCache(*(torch.zeros(t // 16 + 1, 1, 16, D, dtype=torch.float16, device="cuda") for _ in range(2)))
        slots, positions, freqs = ints(np.arange(t)), ints(np.arange(t)), gpu(_freqs(64))
        out = torch.zeros(t, 2, D, dtype=torch.float16, device="cuda")

        def call():
            pk.rotate_rows(config(1, 2), cache, x[:, :2], x[:, 2:3], x[:, 3:], positions, slots, freqs, q_out=out)

        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            x.copy_(gpu(r.standard_normal((t, 4, D)).astype(np.float16)))
            slots.copy_(ints(r.permutation(t)))
            positions.copy_(ints(r.integers(0, 10000, t)))
            graph.replay()
            torch.cuda.synchronize()
            got = [y.clone() for y in (out, cache.K, cache.V)]
            out.zero_()
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (out, cache.K, cache.V)))
