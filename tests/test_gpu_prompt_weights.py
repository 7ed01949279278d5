"""The weights of a token's rows add up to one: where all rows hold the same values, these come back as they are."""

import numpy as np
import pytest

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, draw, gpu

pytestmark = pytest.mark.gpu

# A float16 value just below a power of two (half a step of it is 2^-12 of it) and the largest; a float32 sum of the
# weighted rows, n of them at most, is off by less than n 2^-24, 2^-13 of it here.
VALUES = [1.9990234375, -65504.0]


def _run(q, K, value, pos, sink, window):
    b, hq, t, _ = q.shape
    V = np.full(K.shape, value, np.float16)
    cfg = pk.Config(K.shape[1], hq // K.shape[1], 64, workloads.rotation_signs(3))
    got = pk.sink_window_attend(cfg, gpu(q), gpu(K), gpu(V), pos, sink, window, SCALE).cpu().numpy()
    assert (got == np.float16(value)).all(), f"{(got != np.float16(value)).sum()} of {got.size} values differ"


@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("t", [4, 300, 1100])
def test_weights_of_random_scores(t, value):
    r = np.random.default_rng(t)
    _run(draw(r, 1, 4, t, D), draw(r, 1, 2, 700 + t, D), value, 700, 4, 500)


@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("t", [4, 300, 1100])
def test_weights_that_round_alike(t, value):
    # The first 64 rows score 0; the others score alike, up to 2^6 times their weight: whatever one weight loses to
    # rounding, all of them lose.
    r = np.random.default_rng(t)
    K = np.zeros((1, 2, 700 + t, D), np.float16)
    K[:, :, 64:, 0] = 1
    q = draw(r, 1, 4, t, D)
    q[..., 0] = r.uniform(0, 47, q.shape[:-1])
    _run(q, K, value, 700, 64, 5000)
