"""Plans of pages against the same plan made sequence by sequence in Python: every array, entry for entry."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
from pages import ints, plan

pytestmark = pytest.mark.gpu

NAMES = ("lens", "n_free", "offsets", "counts", "slots", "positions")


def _check(table, free, n_free, lens, counts, page, t, in_place=False):
    print(f"[plan] batch {len(lens)} width {table.shape[1]} pages {len(free)} free {n_free} page {page} t {t}", flush=True)
    want = plan(table, free, n_free, lens, counts, page, t)
    gt, gf, gn, gl, gc = (ints(x) for x in (table, free, [n_free], lens, counts))
    out = pk.PagePlan(gl, gn, ints(np.full(len(lens) + 1, 9)), gc, ints(np.full(t, 9)), ints(np.full(t, 9))) if in_place else None
    got = pk.plan_pages(gt, gf, gn, gl, gc, page, t=t, plan=out)
    for k in NAMES:
        assert np.array_equal(getattr(got, k).cpu().numpy(), want[k]), k
    assert np.array_equal(gt.cpu().numpy(), want["table"]) and np.array_equal(gf.cpu().numpy(), want["free"])
    return want


def _state(r, batch, longest, page, spare, empty=0.0):
    """Sequences in a pool of pages: (table, free, n_free, lens)."""
    lens = r.integers(0, longest + 1, batch)
    lens[r.random(batch) < empty] = 0
    held = -(-lens // page)
    width = max(1, -(-longest // page) + 3)
    pages = int(held.sum()) + spare
    perm = r.permutation(max(pages, 1))
    table = r.integers(-5, 5, (batch, width))
    at = 0
    for b in range(batch):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(max(pages, 1), -3)
    free[:spare] = perm[at:at + spare]
    return table.astype(np.int32), free.astype(np.int32), spare, lens


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 1000, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("page", [1, 7, 16, 100])
def test_a_step(batch, page):
    # Most sequences get one row, some end, some begin; there are pages for all, and for half.
    r = np.random.default_rng(batch + page)
    for spare in (batch + 40, batch // 20):
        table, free, n_free, lens = _state(r, batch, 300, page, spare, empty=0.1)
        counts = np.ones(batch, dtype=np.int64)
        kind = r.random(batch)
        counts[kind < 0.1] = -r.integers(0, 400, (kind < 0.1).sum())
        counts[(kind > 0.9)] = r.integers(0, 60, (kind > 0.9).sum())
        t = int(np.maximum(counts, 0).sum()) + 5
        _check(table, free, n_free, lens, counts, page, t)
        _check(table, free, n_free, lens, counts, page, t, in_place=True)


@pytest.mark.parametrize("t", [1, 4095, 4096, 4097, 20000])
def test_prompts_and_token_arrays_of_all_sizes(t):
    r = np.random.default_rng(t)
    for batch in (1, 5, 1500):
        table, free, n_free, lens = _state(r, batch, 2000, 16, 2000, empty=0.8)
        counts = r.integers(0, 2 * t // batch + 2, batch)  # more than t in all, for some seeds
        _check(table, free, n_free, lens, counts, 16, t)
    table, free, n_free, lens = _state(r, 1, 100, 16, 2000)
    table = np.concatenate((table, np.zeros((1, 2000), np.int32)), 1)
    _check(table, free, n_free, lens, [t], 16, t)


def test_what_is_given_back_is_taken_again_in_the_same_order():
    r = np.random.default_rng(5)
    table, free, n_free, lens = _state(r, 40, 300, 16, 10)
    back = _check(table, free, n_free, lens, -lens, 16, 4)
    assert (back["lens"] == 0).all() and back["n_free"][0] == len(free)
    again = _check(back["table"], back["free"], back["n_free"][0], back["lens"], lens, 16, int(lens.sum()))
    assert np.array_equal(again["table"], table) and again["n_free"][0] == n_free


def test_pages_given_back_serve_the_same_step():
    table = np.array([[4, 2, 0], [0, 0, 0], [1, 3, 0]], np.int32)
    out = _check(table, np.zeros(5, np.int32), 0, [32, 0, 20], [-32, 30, 12], 16, 50)
    assert list(out["table"][1, :2]) == [4, 2] and list(out["counts"]) == [0, 30, 12] and out["n_free"][0] == 0


def test_refused_sequences_keep_what_they_have():
    table = np.arange(12, dtype=np.int32).reshape(4, 3)
    free = np.arange(12, 20, dtype=np.int32)
    # The second would need 2 pages of which 1 is there; the third finds room in its own; the last wants one more.
    out = _check(table, free, 2, [16, 10, 17, 16], [1, 30, 4, 1], 16, 40)
    assert list(out["counts"]) == [1, 0, 4, 0] and list(out["lens"]) == [17, 10, 21, 16]
    # Beyond its table; beyond t.
    out = _check(table, free, 8, [48, 40, 0, 0], [1, 9, 20, 11], 16, 40)
    assert list(out["counts"]) == [0, 0, 20, 0]
    out = _check(table, free, 8, [0, 0, 0, 0], [0, 0, 0, 0], 16, 0)
    assert list(out["offsets"]) == [0] * 5


@pytest.mark.parametrize("n_free", [-4, 0, 3, 8, 100])
def test_values_out_of_range_stay_in_bounds(n_free):
    big, low = 2 ** 31 - 1, -2 ** 31
    table = np.arange(18, dtype=np.int32).reshape(6, 3) % 8
    free = np.arange(8, dtype=np.int32)
    _check(table, free, n_free, [big, low, 5, 30, 48, 1], [low, 3, big, big, -1, 2], 16, 64)
    _check(table, free, n_free, [48] * 6, [low] * 6, 16, 3)
    _check(table, free, n_free, [0] * 6, [big] * 6, 16, 30)


def test_a_step_of_many_pages_of_one_row():
    r = np.random.default_rng(2)
    table, free, n_free, lens = _state(r, 3, 5000, 1, 9000)
    _check(table, free, n_free, lens, [-lens[0], 3, -lens[2] // 2], 1, 100)
    table = np.concatenate((table, np.zeros((3, 4000), np.int32)), 1)
    _check(table, free, n_free, lens, [4000, -lens[1], 3000], 1, 7000)


def test_captured_steps_replay():
    r = np.random.default_rng(9)
    for batch, t in ((70, 200), (70, 6000)):
        table, free, n_free, lens = _state(r, batch, 300, 16, 600)
        state = [ints(x) for x in (table, free, [n_free], lens, np.zeros(batch))]
        gt, gf, gn, gl, gc = state
        out = pk.PagePlan(gl, gn, ints(np.zeros(batch + 1)), ints(np.zeros(batch)), ints(np.zeros(t)), ints(np.zeros(t)))

        def call():
            pk.plan_pages(gt, gf, gn, gl, gc, 16, plan=out)

        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(5):
            now = [x.cpu().numpy() for x in (gt, gf, gn, gl)]
            counts = np.where(r.random(batch) < 0.2, -r.integers(0, 100, batch), r.integers(0, t // batch + 1, batch))
            gc.copy_(ints(counts))
            want = plan(now[0], now[1], now[2][0], now[3], counts, 16, t)
            graph.replay()
            torch.cuda.synchronize()
            for k in NAMES:
                assert np.array_equal(getattr(out, k).cpu().numpy(), want[k]), k
            assert np.array_equal(gt.cpu().numpy(), want["table"]) and np.array_equal(gf.cpu().numpy(), want["free"])


def test_another_stream():
    r = np.random.default_rng(1)
    table, free, n_free, lens = _state(r, 30, 300, 16, 100)
    args = [ints(x) for x in (table, free, [n_free], lens, np.full(30, 20))]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = pk.plan_pages(*args, 16, t=600, stream=stream)
    stream.synchronize()
    want = plan(table, free, n_free, lens, np.full(30, 20), 16, 600)
    for k in NAMES:
        assert np.array_equal(getattr(got, k).cpu().numpy(), want[k]), k


def test_the_widest_batch():
    r = np.random.default_rng(3)
    batch = 65535
    table, free, n_free, lens = _state(r, batch, 40, 16, 5000, empty=0.2)
    counts = np.where(r.random(batch) < 0.1, -lens, 1)
    _check(table, free, n_free, lens, counts, 16, batch)
    _check(table, free, n_free, lens, counts, 16, 4000)
