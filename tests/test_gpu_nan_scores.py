"""Scores that are NaN (a NaN query, a NaN in a key that a token sees) make that token's output NaN, and no other's,
also where no other key is in the token's reach, in the wave's, or in the share of the keys that a block takes."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, attend64, check, draw, gpu, mask_words, tolerance
from oracle import quant

pytestmark = pytest.mark.gpu


def _cfg(hkv, g):
    return pk.Config(hkv, g, 64, workloads.rotation_signs(3))


def _compare(got, q, K, V, visible, half_out, what):
    """got [m][D] of queries q [m][D]: NaN where a visible score is NaN, the attention elsewhere."""
    lost = np.isnan(q.astype(np.float64)).any(1) | (visible & np.isnan(K.astype(np.float64)).any(1)[None]).any(1)
    assert np.isnan(got[lost]).all(), f"{what}: {(~np.isnan(got[lost])).sum()} values are not NaN"
    q_, K_ = np.nan_to_num(q), np.nan_to_num(K)
    want = attend64(q_, K_, V, visible)
    check(got[~lost], want[~lost], tolerance(q_, K_, V, half_out=half_out), what)


def _tree(b, hkv, g, n, t, bits, nan_queries=(), nan_drafts=(), lens=None, own_only=False):
    print(f"[nan tree] batch {b} hkv {hkv} g {g} n {n} t {t} bits {bits} queries {nan_queries} drafts {nan_drafts} "
          f"lens {lens}", flush=True)
    r = np.random.default_rng(n + t)
    cfg, cap = _cfg(hkv, g), max(1, n)
    K, V, q = draw(r, b, hkv, cap, D), draw(r, b, hkv, cap, D), draw(r, b, hkv * g, t, D)
    Kt, Vt = draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    q[:, :, list(nan_queries)] = np.nan
    Kt[:, :, list(nan_drafts), 9] = np.nan
    see = np.eye(t, dtype=bool) if own_only else np.tril(np.ones((t, t), bool))
    words = gpu(np.repeat(mask_words(see)[None], b, 0))
    size = [n] * b if lens is None else list(lens)
    ln = None if lens is None else gpu(np.array(lens, np.int32))
    if bits:
        cache = pk.QuantCache.empty(cfg, b, cap, *bits)
        pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, cap)
        K, V = quant.round_trip(K, bits[0]), quant.round_trip(V, bits[1])
        out = pk.quant_tree_attend(cfg, gpu(q), cache, gpu(Kt), gpu(Vt), n, SCALE, mask=words, lens=ln)
    else:
        out = pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, SCALE, mask=words, lens=ln)
    out = out.cpu().numpy()
    for s in range(b):
        visible = np.concatenate([np.ones((t, size[s]), bool), see], 1)
        for h in range(hkv * g):
            k_ = np.concatenate([K[s, h // g, :size[s]], Kt[s, h // g]])
            v_ = np.concatenate([V[s, h // g, :size[s]], Vt[s, h // g]])
            _compare(out[s, h], q[s, h], k_, v_, visible, False, f"seq {s} head {h}")


FORMS = [(4, 3), (4, 8), (4, 16), (4, 31)]  # (heads, drafts): 16, 32, 64 and 128 rows a block


@pytest.mark.parametrize("bits", [None, (8, 8), (4, 4)])
@pytest.mark.parametrize("n", [0, 70, 3000])  # no cached row, one share of the keys, several
@pytest.mark.parametrize("g,t", FORMS)
def test_a_draft_whose_query_is_nan(g, t, n, bits):
    _tree(2, 2, g, n, t, bits, nan_queries=(1,))


@pytest.mark.parametrize("bits", [None, (8, 8), (4, 4)])
@pytest.mark.parametrize("g,t", FORMS)
def test_a_draft_that_sees_only_a_nan_key(g, t, bits):
    _tree(2, 2, g, 0, t, bits, nan_drafts=(0, t - 1), own_only=True)


@pytest.mark.parametrize("bits", [None, (8, 8), (4, 4)])
@pytest.mark.parametrize("g,t", [(4, 1), (16, 2), (16, 4), (16, 8)])
def test_a_share_that_holds_only_nan_keys(g, t, bits):
    # Shares are cut by n: the last one of these short sequences has the drafts alone.
    _tree(2, 1, g, 3000, t, bits, nan_drafts=range(t), lens=(128, 256))


def _window(b, hkv, g, pos, t, sink, window, nan_queries=(), nan_keys=(), starts=None):
    print(f"[nan window] batch {b} hkv {hkv} g {g} pos {pos} t {t} sink {sink} window {window} queries {nan_queries} "
          f"keys {nan_keys} starts {starts}", flush=True)
    r = np.random.default_rng(pos + t)
    K, V, q = draw(r, b, hkv, pos + t, D), draw(r, b, hkv, pos + t, D), draw(r, b, hkv * g, t, D)
    q[:, :, list(nan_queries)] = np.nan
    K[:, :, list(nan_keys), 77] = np.nan
    st = None if starts is None else gpu(np.array(starts, np.int32))
    got = pk.sink_window_attend(_cfg(hkv, g), gpu(q), gpu(K), gpu(V), pos, sink, window, SCALE, starts=st).cpu().numpy()
    for s in range(b):
        first = pos if starts is None else starts[s]
        n = first + t
        p, j = np.arange(first, n)[:, None], np.arange(n)[None]
        visible = (j <= p) & ((j < sink) | (j > p - window))
        for h in range(hkv * g):
            _compare(got[s, h], q[s, h], K[s, h // g, :n], V[s, h // g, :n], visible, True, f"seq {s} head {h}")


@pytest.mark.parametrize("b,hkv,g,pos,t,window", [
    (1, 2, 4, 0, 2, 64), (2, 2, 4, 700, 1, 64), (2, 2, 4, 3000, 2, 2048), (1, 2, 4, 3000, 8, 2048),
    (1, 2, 4, 3000, 16, 2048), (1, 2, 4, 3000, 40, 2048), (1, 1, 2, 0, 300, 100), (1, 1, 2, 3000, 1100, 100)])
def test_a_token_whose_query_is_nan(b, hkv, g, pos, t, window):
    _window(b, hkv, g, pos, t, 4, window, nan_queries=(0, t // 2))


@pytest.mark.parametrize("pos,t", [(700, 1), (700, 6), (700, 40), (0, 300), (3000, 1100)])
def test_a_token_that_sees_only_a_nan_key(pos, t):
    _window(2, 2, 4, pos, t, 0, 1, nan_keys=(pos, pos + t // 2))


@pytest.mark.parametrize("t", [1, 8, 16, 40, 300])
def test_a_nan_key_in_the_first_row_of_a_prompt(t):
    _window(2, 2, 4, 0, t, 0, 20, nan_keys=(0,))


@pytest.mark.parametrize("g", [1, 8, 16])
def test_a_token_whose_own_key_is_nan_and_alone_in_its_share(g):
    # Rows 0 .. 127 in one share of the keys, the token's own in the next.
    _window(2, 1, g, 3000, 1, 0, 4000, nan_keys=(128, 256), starts=(128, 256))


@pytest.mark.parametrize("kb,vb", [(8, 8), (4, 4)])
@pytest.mark.parametrize("k", [1, 16, 64, 65, 300])
@pytest.mark.parametrize("what", ["query", "window row", "only row"])
def test_listed_rows(what, k, kb, vb):
    print(f"[nan listed] {what} k {k} bits {kb} {vb}", flush=True)
    b, hkv, g, n = 2, 2, 4, 400
    r = np.random.default_rng(k)
    cfg, win = _cfg(hkv, g), pk.Window(3, 3, n, n + 9)
    K, V, q = draw(r, b, hkv, n, D), draw(r, b, hkv, n, D), draw(r, b, hkv * g, D)
    Kw, Vw = draw(r, b, hkv, 16, D), draw(r, b, hkv, 16, D)
    idx = np.stack([np.sort(r.permutation(n - 3)[:k]) for _ in range(b * hkv * g)]).reshape(b, hkv * g, k).astype(np.int32)
    if what == "query":
        q[:, 1::2] = np.nan
    else:
        Kw[:, 1, 5, 40] = np.nan  # slot 5 of one KV head: a Local row
    if what == "only row":
        idx[:] = -1
        win = pk.Window(0, 0, n - 11, n - 10)
        Kw[:, 1, (n - 11) % 16, 40] = np.nan
    cache = pk.QuantCache.empty(cfg, b, n, kb, vb)
    pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, n)
    K, V = quant.round_trip(K, kb), quant.round_trip(V, vb)
    plain = pk.quant_attend(cfg, gpu(q), cache, gpu(idx), SCALE).cpu().numpy()
    tiered = pk.quant_tiered_attend(cfg, gpu(q), gpu(Kw), gpu(Vw), cache, gpu(idx), win, SCALE).cpu().numpy()
    slots = [pk.window_slot(x, win.sink_len, 16) for x in
             list(range(win.sink_len)) + list(range(win.dense_begin, win.dense_end))]
    for s in range(b):
        for h in range(hkv * g):
            rows = idx[s, h][idx[s, h] >= 0]
            for got, first, dense in ((plain, 0, []), (tiered, win.retr_begin, slots)):
                k_ = np.concatenate([K[s, h // g, first + rows], Kw[s, h // g, dense].astype(np.float64)])
                v_ = np.concatenate([V[s, h // g, first + rows], Vw[s, h // g, dense].astype(np.float64)])
                if len(k_) == 0:
                    assert not got[s, h].any()
                    continue
                _compare(got[s, h][None], q[s, h][None], k_, v_, np.ones((1, len(k_)), bool), False, f"seq {s} head {h}")
