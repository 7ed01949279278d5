"""Many rows that weigh next to nothing beside one: what their weights lose to float16 stays in the stated bounds.

One row scores 0 and holds 0, the n others score alike, log2 of their weight from 0 to -40, and hold 1: a token's output
is n w / (1 + n w).  Scores are single exact products, at most A = 28 here; as in tolerance() a weight is off by
2^-22 A (its product with log2 e, the subtraction) and 2^-20 (the exponential, the sums) of itself, the output by
twice that of itself.  P is at least 2^8 for the largest weight; its two float16 parts leave 2^-22 of it or 2^-25,
which is 2^-33 of the largest: n 2^-33 for the output.  One part leaves 2^-11 of it or as much, and the sum takes the
same; a float16 output adds half a step, 2^-11 of it or 2^-25."""

import numpy as np
import pytest

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, gpu
from oracle import quant

pytestmark = pytest.mark.gpu

OWN = 2 * (28 * 2.0 ** -22 + 2.0 ** -20)


def _inputs(hkv, g, n, t, seed):
    r = np.random.default_rng(seed)
    K, V = np.zeros((2, 1, hkv, n + 1, D), np.float16)
    K[:, :, :, 0], V[:] = -1, 1
    at = int(r.integers(0, n + 1))
    K[:, :, at], V[:, :, at] = 0, 0
    q = np.zeros((1, hkv * g, t, D), np.float16)
    q[..., 0] = r.uniform(0, 40, q.shape[:-1]) / (SCALE * 1.4426950408889634)
    w = np.exp(-SCALE * q[..., 0].astype(np.float64))
    return q, K, V, n * w / (1 + n * w)


def _check(got, want, tol):
    off = np.abs(got.astype(np.float64) - want[..., None]) / tol[..., None]
    assert off.max() <= 1, f"off by {off.max():.3g} of what is allowed"


@pytest.mark.parametrize("bits", [None, (8, 8)])
@pytest.mark.parametrize("n", [100, 5000, 60000])
@pytest.mark.parametrize("g,t", [(4, 3), (4, 8), (4, 16), (4, 31)])
def test_drafts(g, t, n, bits):
    print(f"[small weights] drafts g {g} t {t} n {n} bits {bits}", flush=True)
    q, K, V, want = _inputs(2, g, n, t, n + t)
    cfg = pk.Config(2, g, 64, workloads.rotation_signs(3))
    nothing = gpu(np.zeros((1, t), np.int64))  # the drafts see no draft
    Kt = gpu(np.zeros((1, 2, t, D), np.float16))
    if bits:
        cache = pk.QuantCache.empty(cfg, 1, n + 1, *bits)
        pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, n + 1)
        assert (quant.round_trip(K[:, :, :9], 8) == K[:, :, :9]).all()
        out = pk.quant_tree_attend(cfg, gpu(q), cache, Kt, Kt, n + 1, SCALE, mask=nothing)
    else:
        out = pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), Kt, Kt, n + 1, SCALE, mask=nothing)
    _check(out.cpu().numpy(), want, OWN * want + n * 2.0 ** -33)


@pytest.mark.parametrize("n,t", [(100, 1), (5000, 4), (60000, 16), (5000, 300), (60000, 1100)])
def test_windows(n, t):
    print(f"[small weights] window n {n} t {t}", flush=True)
    q, K, V, want = _inputs(2, 4, n, t, n + t)
    cfg = pk.Config(2, 4, 64, workloads.rotation_signs(3))
    # The new tokens' rows: keys that nobody reaches, for the sinks are all that the tokens see but their own.
    K = np.concatenate([K, np.zeros((1, 2, t, D), np.float16)], 2)
    V = np.concatenate([V, np.zeros((1, 2, t, D), np.float16)], 2)
    out = pk.sink_window_attend(cfg, gpu(q), gpu(K), gpu(V), n + 1, n + 1, 1, SCALE).cpu().numpy()
    w = np.exp(-SCALE * q[..., 0].astype(np.float64))
    want = n * w / (2 + n * w)  # a token's own row scores 0 and holds 0 as well
    _check(out, want, (OWN + 2.0 ** -10) * want + n * 2.0 ** -33 + 2.0 ** -25)
