"""Float64 attention of several new tokens and the tolerance its kernels are held to."""

import numpy as np
import torch

D = 128
SCALE = D ** -0.5


def draw(r, *shape, law=1.0):
    return (law * r.standard_normal(shape)).astype(np.float16)


def attend64(q, K, V, visible, scale=SCALE):
    """softmax(scale q K^T) V over the visible pairs; q [m][D], K and V [n][D], visible [m][n]; zeros where none."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    if K.shape[0] == 0:
        return np.zeros((q.shape[0], D))
    s = np.where(visible, scale * (q @ K.T), -np.inf)
    top = s.max(1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    p = np.where(visible, p, 0.0)
    total = p.sum(1, keepdims=True)
    return np.where(total > 0, p @ np.where(visible.any(0)[:, None], V, 0.0), 0.0) / np.where(total > 0, total, 1.0)


def tolerance(q, K, V, scale=SCALE, half_out=False):
    """Largest error of an output.

    float32 out: a score is a sum of 128 exact products with at most 128 roundings to float32 (2^-24 of a partial sum,
    itself at most A = scale sum |q k|); roundings are independent, so 4 sqrt(128) 2^-24 A bounds what they add up to,
    and 2^-22 A the products with the scale and the subtraction of the maximum.  A weight is then off by that and 2^-20
    (the exponential, the split of P, the sums), an output by twice a weight's error times the largest value, and the
    same rounding of its own sums.
    float16 out adds P's rounding (2^-11 of each weight) and the output's (2^-11)."""
    q, K, V = (np.abs(np.asarray(x, dtype=np.float64)) for x in (q, K, V))
    if K.shape[0] == 0:
        return 0.0
    A = abs(scale) * (q @ K.T).max()
    rel = 2 * ((4 * np.sqrt(128) * 2.0 ** -24 + 2.0 ** -22) * A + 2.0 ** -20)
    return (rel + (2.0 ** -10 if half_out else 0.0)) * V.max()


def gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def check(got, want, tol, what):
    off = np.abs(np.asarray(got, dtype=np.float64) - want).max() if want.size else 0.0
    assert np.isfinite(got).all() and off <= tol, f"{what}: off by {off:.3g}, allowed {tol:.3g}"


def random_tree(r, t):
    """Ancestor masks bool [t][t] of a random tree: a token sees itself and the path to its root."""
    see = np.zeros((t, t), dtype=bool)
    for i in range(t):
        parent = int(r.integers(-1, i)) if i else -1
        if parent >= 0:
            see[i] = see[parent]
        see[i, i] = True
    return see


def mask_words(see):
    t = see.shape[-1]
    return (see.astype(np.uint64) << np.arange(t, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)
