"""Paged caches for tests: a step's plan sequence by sequence, rotation and attention in 64 bits."""

import numpy as np
import torch

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE

MOST_ROWS = 2 ** 30 - 1


def config(hkv, g):
    return pk.Config(hkv, g, 1, workloads.rotation_signs(3))


def plan(table, free, n_free, lens, counts, page, t):
    """pariskv_plan_pages in Python: a dict of its arrays after the step (int32)."""
    table, free = table.copy(), free.copy()
    batch, width = table.shape
    room = min(width * page, MOST_ROWS)
    lens = [min(max(int(x), 0), room) for x in lens]
    counts = [int(x) for x in counts]
    begin = min(max(int(n_free), 0), len(free))
    back = [table[b, j] for b in range(batch) if counts[b] < 0
            for j in range(-(-max(lens[b] + counts[b], 0) // page), -(-lens[b] // page))]
    for i, x in enumerate(reversed(back)):
        if begin + i < len(free):
            free[begin + i] = x
    top = min(begin + len(back), len(free))
    out = dict(offsets=[0], counts=[], lens=[], slots=np.full(t, -1), positions=np.full(t, -1))
    wanted = taken = at = 0
    for b in range(batch):
        n = max(counts[b], 0)
        total = max(lens[b] + counts[b], 0)
        have, want = -(-lens[b] // page), -(-total // page)
        ok = n > 0 and total <= room and at + n <= t
        if ok:
            first = wanted
            wanted += want - have
            ok = want == have or wanted <= top
        if ok:
            for j in range(have, want):
                table[b, j] = free[top - 1 - first - (j - have)]
            taken += want - have
            rows = np.arange(lens[b], total)
            out["slots"][at:at + n] = table[b, rows // page] * page + rows % page
            out["positions"][at:at + n] = rows
        out["counts"].append(n if ok else 0)
        out["lens"].append(total if ok or counts[b] < 0 else lens[b])
        at += n
        out["offsets"].append(min(at, t))
    out.update(table=table, free=free, n_free=[top - taken])
    return {k: np.asarray(v, dtype=np.int32) for k, v in out.items()}


def rotate64(x, positions, freqs, weight, eps, pairs):
    """x [t][heads][D] normalised and rotated in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if freqs is None:
        return x
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(freqs, dtype=np.float64)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    half = len(freqs)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


def attend64(q, K, V, positions, there, scale, cap, slopes):
    """One KV head: q [m][g][D] at positions [m] over K, V [n][D] of which there [n] are there, in 64 bits; zeros where a
    token attends nothing."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    m, g = q.shape[:2]
    j = np.arange(K.shape[0])
    seen = (j[None] <= np.asarray(positions)[:, None]) & there[None]
    if K.shape[0] == 0:
        return np.zeros((m, g, D))
    K, V = np.where(there[:, None], K, 0.0), np.where(there[:, None], V, 0.0)
    s = scale * np.einsum("mgd,nd->mgn", q, K)
    if cap > 0:
        s = cap * np.tanh(s / cap)
    if slopes is not None:
        s = s + np.asarray(slopes, dtype=np.float64)[None, :, None] * (j[None] - np.asarray(positions)[:, None])[:, None]
    s = np.where(seen[:, None], s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdims=True)
    return np.where(total > 0, np.einsum("mgn,nd->mgd", p, V) / np.where(total > 0, total, 1.0), 0.0)


def tolerance(q, K, V, scale, cap=0.0, slopes=None):
    """Largest error of an output: as new_tokens.tolerance for float16 outputs, with what the score's shape adds: with
    scores A at most, 2^-21 of the cap (the header's bound: the tanh's exponential and reciprocal) and, with a bias B at
    most, the rounding of its product and of its sum with the score, 2^-23 (A + B) for those within 40 of the largest (the
    others weigh less than 2^-57); a weight is off by as much, an output by twice that."""
    q, K, V = (np.abs(np.asarray(x, dtype=np.float64)) for x in (q, K, V))
    if K.shape[0] == 0:
        return 0.0
    A = abs(scale) * (q.reshape(-1, D) @ K.T).max()
    rel = 2 * ((4 * np.sqrt(128) * 2.0 ** -24 + 2.0 ** -22) * A + 2.0 ** -20) + 2.0 ** -10
    rel += 2 * 2.0 ** -21 * cap
    if slopes is not None:
        top = min(cap, A) if cap > 0 else A
        rel += 2 * 2.0 ** -23 * (2 * top + 40 + top)
    return rel * V.max()


class Pool:
    """Sequences of given lengths in a pool of scattered pages; every row that none of them has holds NaN."""

    def __init__(self, r, hkv, lens, page, law=1.0, spare=3, extra_width=1):
        held = [-(-n // page) for n in lens]
        self.page, self.lens = page, lens
        pages = sum(held) + spare
        perm = r.permutation(pages)
        self.K = np.full((pages, hkv, page, D), np.nan, dtype=np.float16)
        self.V = self.K.copy()
        self.table = np.full((len(lens), max(held + [0]) + extra_width), -7, dtype=np.int32)
        self.rows = []
        at = 0
        for b, n in enumerate(lens):
            mine = perm[at:at + held[b]]
            at += held[b]
            self.table[b, :held[b]] = mine
            j = np.arange(n)
            k, v = ((law * r.standard_normal((n, hkv, D))).astype(np.float16) for _ in range(2))
            v = (v / law).astype(np.float16)
            self.K[mine[j // page], :, j % page] = k
            self.V[mine[j // page], :, j % page] = v
            self.rows.append((k, v))

    def cache(self):
        return pk.PagedCache(torch.from_numpy(self.K).cuda(), torch.from_numpy(self.V).cuda())


def ints(x):
    return torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
