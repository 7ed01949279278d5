"""GPU parity of the attention of new tokens over a sliding window and the first tokens, against float64."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, attend64, check, draw, gpu, tolerance

pytestmark = pytest.mark.gpu


def _cfg(hkv, g):
    return pk.Config(hkv, g, 64, workloads.rotation_signs(3))


def _run(b, hkv, g, pos, t, sink, window, starts=None, counts=None, scale=SCALE, seed=0, slack=3):
    """One call checked in every output; cache rows behind a sequence's last token hold NaN, and rows of out behind its
    tokens have to stay as they were."""
    print(f"[sink] batch {b} hkv {hkv} g {g} pos {pos} t {t} sink {sink} window {window} starts {starts} "
          f"counts {counts}", flush=True)
    r = np.random.default_rng(seed)
    cap = pos + t + slack
    K, V, q = draw(r, b, hkv, cap, D), draw(r, b, hkv, cap, D), draw(r, b, hkv * g, t, D)
    first = [pos] * b if starts is None else [min(max(x, 0), pos) for x in starts]
    real = [t] * b if counts is None else [min(max(x, 0), t) for x in counts]
    for s in range(b):
        K[s, :, first[s] + real[s]:] = V[s, :, first[s] + real[s]:] = np.nan
        q[s, :, real[s]:] = np.nan
    out = torch.full((b, hkv * g, t, D), 7.0, dtype=torch.float16, device="cuda")
    st = None if starts is None else gpu(np.array(starts, np.int32))
    ct = None if counts is None else gpu(np.array(counts, np.int32))
    got = pk.sink_window_attend(_cfg(hkv, g), gpu(q), gpu(K), gpu(V), pos, sink, window, scale, starts=st, counts=ct,
                                out=out).cpu().numpy()
    for s in range(b):
        n, m = first[s] + real[s], real[s]
        assert (got[s, :, m:] == 7).all(), f"seq {s}: padding was written"
        if m == 0:
            continue
        p, j = np.arange(first[s], n)[:, None], np.arange(n)[None]
        visible = (j <= p) & ((j < sink) | (j > p - window))
        for h in range(hkv * g):
            k_, v_ = K[s, h // g, :n], V[s, h // g, :n]
            want = attend64(q[s, h, :m], k_, v_, visible, scale)
            check(got[s, h, :m], want, tolerance(q[s, h, :m], k_, v_, scale, half_out=True), f"seq {s} head {h}")


@pytest.mark.parametrize("t", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 257, 500])
@pytest.mark.parametrize("sink,window", [(0, 1), (4, 64), (128, 100)])
def test_prompts(t, sink, window):
    _run(1, 2, 2, 0, t, sink, window, seed=t)


@pytest.mark.parametrize("pos,t", [(1, 1), (63, 1), (700, 1), (700, 16), (700, 17), (701, 128), (333, 300), (5000, 3)])
@pytest.mark.parametrize("sink,window", [(0, 64), (4, 63), (128, 512), (1, 1), (0, 100000), (2000, 10)])
def test_later_chunks(pos, t, sink, window):
    _run(1, 1, 4, pos, t, sink, window, seed=pos + t)


@pytest.mark.parametrize("g", [1, 3, 7, 16])
@pytest.mark.parametrize("t", [1, 5, 140])
def test_heads_per_kv_head(g, t):
    _run(2, 3, g, 400, t, 16, 200, seed=g)


@pytest.mark.parametrize("t", [1, 4, 300])
def test_sequences_that_begin_at_different_positions(t):
    _run(5, 2, 4, 900, t, 8, 128, starts=[0, 900, 450, -3, 1000], seed=t)


@pytest.mark.parametrize("t", [2, 16, 260])
def test_padded_prompts(t):
    _run(5, 2, 2, 0, t, 4, 50, counts=[0, 1, t, t - 1, t + 9], seed=t)
    _run(4, 1, 3, 600, t, 4, 50, starts=[600, 0, 30, 599], counts=[t, 0, 1, -5], seed=t)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.4])
@pytest.mark.parametrize("t", [3, 150])
def test_scales(scale, t):
    _run(1, 2, 2, 100, t, 4, 64, scale=scale, seed=1)


def test_more_than_eight_kv_heads_and_sequences():
    _run(3, 9, 2, 50, 130, 4, 64, seed=4)
    _run(5, 7, 1, 300, 2, 4, 64, seed=4)


def test_both_forms_agree():
    # 4 tokens by the form whose blocks share the keys, the same among 1100 by the other.
    b, hkv, g, pos, t = 2, 2, 4, 1000, 1100
    r = np.random.default_rng(3)
    K, V, q = draw(r, b, hkv, pos + t, D), draw(r, b, hkv, pos + t, D), draw(r, b, hkv * g, t, D)
    cfg = _cfg(hkv, g)
    whole = pk.sink_window_attend(cfg, gpu(q), gpu(K), gpu(V), pos, 8, 300, SCALE).cpu().numpy()
    part = pk.sink_window_attend(cfg, gpu(q[:, :, :4]), gpu(K), gpu(V), pos, 8, 300, SCALE).cpu().numpy()
    for s in range(b):
        for h in range(hkv * g):
            tol = tolerance(q[s, h], K[s, h // g], V[s, h // g], half_out=True)
            check(whole[s, h, :4], part[s, h].astype(np.float64), 2 * tol, f"seq {s} head {h}")


def test_captured_calls_replay():
    b, hkv, g, pos = 3, 2, 4, 1500
    r = np.random.default_rng(9)
    cfg = _cfg(hkv, g)
    for t in (1, 200):
        q, K, V = (gpu(x) for x in (draw(r, b, hkv * g, t, D), draw(r, b, hkv, pos + t, D), draw(r, b, hkv, pos + t, D)))
        starts = torch.zeros(b, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(q)
        ws = torch.empty(pk.sink_window_workspace_size(cfg, b, pos, t, 4, 600), dtype=torch.uint8, device="cuda")

        def call():
            pk.sink_window_attend(cfg, q, K, V, pos, 4, 600, SCALE, starts=starts, out=out, workspace=ws)

        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(4):
            starts.copy_(gpu(r.integers(0, pos + 1, b).astype(np.int32)))
            q.copy_(gpu(draw(r, b, hkv * g, t, D)))
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.zero_()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got, out)


@pytest.mark.parametrize("b,hkv,g,pos,t,window", [
    (1, 2, 4, 3000, 1, 2048), (1, 1, 16, 3000, 2, 2048), (2, 1, 8, 4000, 8, 3000), (1, 2, 4, 4000, 40, 4000),
    (1, 1, 7, 5000, 19, 4500), (1, 1, 2, 6000, 300, 4000), (9, 1, 1, 2500, 70, 2500), (1, 1, 1, 9000, 1000, 9000)])
def test_long_windows_with_shared_keys(b, hkv, g, pos, t, window):
    # Blocks share a sequence's keys: 16, 32, 64 and 128 rows of it a block, and more.
    _run(b, hkv, g, pos, t, 100, window, seed=t)
    _run(b, hkv, g, pos, t, 0, window, seed=t, starts=list(np.linspace(0, pos, b).astype(int)),
         counts=[max(1, t - i) for i in range(b)])


@pytest.mark.parametrize("b,hkv,g,pos,t,window", [(1, 2, 4, 200, 1, 64), (2, 4, 4, 300, 9, 30), (40, 8, 2, 64, 33, 500)])
def test_short_windows_in_one_launch(b, hkv, g, pos, t, window):
    _run(b, hkv, g, pos, t, 5, window, seed=t, starts=[(7 * i) % (pos + 1) for i in range(b)],
         counts=[(5 * i) % (t + 1) for i in range(b)])


@pytest.mark.parametrize("b,hkv,g,pos,t,sink,window", [
    (1, 1, 4, 3000, 4, 40, 2000), (1, 2, 4, 3000, 8, 40, 2000), (2, 1, 4, 3000, 16, 40, 2000),
    (1, 1, 4, 3000, 40, 0, 2000), (64, 8, 4, 120, 4, 5, 60), (64, 8, 4, 120, 8, 0, 60),  # few tokens
    (1, 2, 2, 500, 300, 40, 100), (2, 1, 2, 0, 500, 3, 64), (1, 1, 2, 0, 200, 0, 1000)])  # prompt form
def test_rows_that_are_not_finite_reach_only_tokens_that_see_them(b, hkv, g, pos, t, sink, window):
    print(f"[sink] not finite: batch {b} hkv {hkv} g {g} pos {pos} t {t} sink {sink} window {window}", flush=True)
    r = np.random.default_rng(pos + t)
    n = pos + t
    K, V, q = draw(r, b, hkv, n, D), draw(r, b, hkv, n, D), draw(r, b, hkv * g, t, D)
    # Rows that some tokens see and some do not: the last token's own, one in the middle, the
    # first token's oldest, and a row behind the sinks.
    values = {n - 1: np.inf, pos + t // 2: np.nan, max(sink, pos - window + 1): -np.inf, sink: np.inf}
    bad = V.copy()
    for i, (j, x) in enumerate(values.items()):
        bad[:, :, j, 5 + 30 * i] = bad[:, :, j, 127] = x
    odd = ~np.isfinite(bad)
    V[odd] = 0
    lost, badk = pos + t // 3, K.copy()  # a row whose scores are NaN
    badk[:, :, lost, 77], K[:, :, lost] = np.nan, 0
    got = pk.sink_window_attend(_cfg(hkv, g), gpu(q), gpu(badk), gpu(bad), pos, sink, window, SCALE).cpu().numpy()
    p, j = np.arange(pos, n)[:, None], np.arange(n)[None]
    visible = (j <= p) & ((j < sink) | (j > p - window))
    assert not visible[:, list(values)].all(0).all(), "some of the rows are hidden from some token"
    dead = visible[:, lost]
    for s in range(0, b, 21):
        for h in range(hkv * g):
            x, v = got[s, h].astype(np.float32), bad[s, h // g].astype(np.float32)
            assert np.isnan(x[dead]).all()
            odds = np.stack([np.where(np.isfinite(v[m]), 0, v[m]).sum(0) for m in visible])
            hit = (odds != 0) & ~dead[:, None]
            assert np.array_equal(x[hit], odds[hit], equal_nan=True)
            k_, v_ = K[s, h // g], V[s, h // g]
            fine = ~hit & ~dead[:, None]
            want = attend64(q[s, h], k_, v_, visible)
            check(got[s, h][fine], want[fine], tolerance(q[s, h], k_, v_, half_out=True), f"seq {s} head {h}")
