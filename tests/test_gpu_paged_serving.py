"""A server's steps over a paged cache, as they would run: pages planned, rows rotated and written, attended, captured."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
from new_tokens import D, SCALE, check, gpu
from pages import attend64, config, ints, plan, rotate64, tolerance

pytestmark = pytest.mark.gpu

EPS, ROT = 1e-6, 64


class Server:
    """One layer's paged cache and the float64 record of what every sequence holds."""

    def __init__(self, r, hkv, g, page, batch, pages, width):
        self.r, self.hkv, self.g, self.page, self.batch = r, hkv, g, page, batch
        self.cfg = config(hkv, g)
        self.cache = pk.PagedCache.empty(self.cfg, pages, page)
        self.cache.K.fill_(float("nan"))
        self.cache.V.fill_(float("nan"))
        self.table, self.free = ints(np.zeros((batch, width))), ints(r.permutation(pages))
        self.n_free, self.lens = ints([pages]), ints(np.zeros(batch))
        self.freqs = gpu(np.array([10000.0 ** (-2 * i / ROT) for i in range(ROT // 2)], dtype=np.float32))
        self.weights = [gpu((1 + 0.2 * r.standard_normal(D)).astype(np.float32)) for _ in range(2)]
        self.rows = [(np.zeros((0, hkv, D)), np.zeros((0, hkv, D))) for _ in range(batch)]

    def state(self):
        return [x.cpu().numpy() for x in (self.table, self.free, self.n_free, self.lens)]

    def launch(self, x, counts, most, out, plan_, workspace):
        """One step of tokens x [t][Hq + 2 Hkv][D] on the GPU."""
        hq, hkv = self.hkv * self.g, self.hkv
        pk.plan_pages(self.table, self.free, self.n_free, self.lens, counts, self.page, plan=plan_)
        q = pk.rotate_rows(self.cfg, self.cache, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], plan_.positions, plan_.slots,
                           self.freqs, *self.weights, eps=EPS)
        return pk.paged_attend(self.cfg, q, self.cache, self.table, plan_.lens, plan_.offsets, SCALE, counts=plan_.counts,
                               max_tokens=most, out=out, workspace=workspace)

    def verify(self, before, x, counts, out):
        """A step's outputs against float64, and the record brought up to date."""
        hq, hkv, t = self.hkv * self.g, self.hkv, x.shape[0]
        want = plan(*before[:2], before[2][0], before[3], counts, self.page, t)
        for k, got in zip(("table", "free", "n_free", "lens"), self.state()):
            assert np.array_equal(got, want[k]), k
        f = self.freqs.cpu().numpy()
        qw, kw = (w.cpu().numpy() for w in self.weights)
        kept = np.ones(t, dtype=bool)
        for b in range(self.batch):
            lo, m = want["offsets"][b], want["counts"][b]
            K, V = self.rows[b]
            if counts[b] < 0:
                n = max(len(K) + counts[b], 0)
                self.rows[b] = K[:n], V[:n]
                continue
            if m == 0:
                continue
            kept[lo:lo + m] = False
            p = np.arange(len(K), len(K) + m)
            rows = x[lo:lo + m]
            # What the cache and the attention hold are float16 values.
            q = rotate64(rows[:, :hq], p, f, qw, EPS, False).astype(np.float16)
            K = np.concatenate((K, rotate64(rows[:, hq:hq + hkv], p, f, kw, EPS, False).astype(np.float16)))
            V = np.concatenate((V, rows[:, hq + hkv:]))
            self.rows[b] = K, V
            for h in range(hkv):
                qh = q.reshape(m, hkv, self.g, D)[:, h]
                ref = attend64(qh, K[:, h], V[:, h], p, np.ones(len(K), bool), SCALE, 0.0, None)
                # The kernel's own float16 rows may be the next value where these lie near a middle: a query and a key each
                # off by a step, 2^-10 of a value, make a score off by 2^-9 of sum |q k| at most.
                A = SCALE * (np.abs(qh.astype(np.float64)).reshape(-1, D) @ np.abs(K[:, h].astype(np.float64)).T).max()
                tol = tolerance(qh, K[:, h], V[:, h], SCALE) + 2 * 2.0 ** -9 * A * np.abs(V[:, h]).max()
                check(out[lo:lo + m].reshape(m, hkv, self.g, D)[:, h], ref, tol, f"seq {b} head {h}")
        assert (out[kept] == 7).all()


def _tokens(r, t, hkv, g):
    return r.standard_normal((t, hkv * g + 2 * hkv, D)).astype(np.float16)


def _counts(r, lens, t, step):
    """Prompts first, then single tokens; some sequences end, some take rows back, new ones begin in their place."""
    counts = np.ones(len(lens), dtype=np.int64)
    for b, n in enumerate(lens):
        if n == 0:
            counts[b] = r.integers(0, t // len(lens)) if step % 2 == 0 else 0
        elif r.random() < 0.15:
            counts[b] = -n
        elif r.random() < 0.15:
            counts[b] = -r.integers(1, 9)
    return counts


@pytest.mark.parametrize("hkv,g,page", [(2, 4, 16), (1, 7, 48), (3, 2, 1)])
def test_steps_of_a_server(hkv, g, page):
    r = np.random.default_rng(page)
    batch, t = 9, 9 * 40
    s = Server(r, hkv, g, page, batch, 40 * (96 // page), -(-300 // page))
    for step in range(10):
        print(f"[serve] hkv {hkv} g {g} page {page} step {step}", flush=True)
        before = s.state()
        counts = _counts(r, before[3], t, step)
        x = _tokens(r, t, hkv, g)
        out = torch.full((t, hkv * g, D), 7.0, dtype=torch.float16, device="cuda")
        plan_ = pk.PagePlan(s.lens, s.n_free, *(ints(np.zeros(n)) for n in (batch + 1, batch, t, t)))
        s.launch(gpu(x), ints(counts), max(int(counts.max()), 1), out, plan_, None)
        s.verify(before, x, counts, out.cpu().numpy())


@pytest.mark.parametrize("most", [1, 4, 40])
def test_a_captured_step_serves_a_generation(most):
    # One graph of the three calls; what changes between the replays is in the arrays.
    r = np.random.default_rng(most)
    hkv, g, page, batch = 2, 4, 16, 6
    t = batch * most
    s = Server(r, hkv, g, page, batch, 120, 40)
    x, counts = gpu(_tokens(r, t, hkv, g)), ints(np.zeros(batch))
    out = torch.full((t, hkv * g, D), 7.0, dtype=torch.float16, device="cuda")
    plan_ = pk.PagePlan(s.lens, s.n_free, *(ints(np.zeros(n)) for n in (batch + 1, batch, t, t)))
    ws = torch.empty(pk.paged_workspace_size(s.cfg, batch, t, most), dtype=torch.uint8, device="cuda")
    s.launch(x, counts, most, out, plan_, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.launch(x, counts, most, out, plan_, ws)
    for step in range(12):
        before = s.state()
        now = np.where(r.random(batch) < 0.1, -r.integers(1, 30, batch), r.integers(0, most + 1, batch))
        host = _tokens(r, t, hkv, g)
        x.copy_(gpu(host))
        counts.copy_(ints(now))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        s.verify(before, host, now, out.cpu().numpy())


def test_chunks_of_a_prompt_and_the_whole_prompt_agree():
    r = np.random.default_rng(5)
    hkv, g, page, n = 2, 4, 16, 500
    x = _tokens(r, n, hkv, g)
    whole = Server(r, hkv, g, page, 1, 64, 40)
    parts = Server(r, hkv, g, page, 1, 64, 40)
    parts.weights = whole.weights
    outs = []
    for s, sizes in ((whole, [n]), (parts, [100, 1, 3, 200, 196])):
        got, at = [], 0
        for m in sizes:
            before = s.state()
            out = torch.full((m, hkv * g, D), 7.0, dtype=torch.float16, device="cuda")
            plan_ = pk.PagePlan(s.lens, s.n_free, *(ints(np.zeros(k)) for k in (2, 1, m, m)))
            s.launch(gpu(x[at:at + m]), ints([m]), m, out, plan_, None)
            s.verify(before, x[at:at + m], np.array([m]), out.cpu().numpy())
            got.append(out)
            at += m
        outs.append(torch.cat(got))
    # Keys and queries are the same values in both, so the outputs differ by less than both tolerances.
    K, V = whole.rows[0]
    diff = (outs[0].double() - outs[1].double()).abs().max().item()
    tol = max(tolerance(np.concatenate([np.asarray(K[:, h])[:, None]] * g, 1), K[:, h], V[:, h], SCALE) for h in range(hkv))
    assert diff <= 2 * tol


def test_a_page_pool_serves_the_other_operators():
    # A dense cache [batch][Hkv][capacity][D] as pages of `capacity` rows: rows written through slots are read by the
    # attention over a dense cache.
    r = np.random.default_rng(6)
    hkv, g, cap, batch, n = 2, 4, 64, 3, 50
    cfg = config(hkv, g)
    cache = pk.PagedCache.empty(cfg, batch, cap)
    x = _tokens(r, batch * n, hkv, g)
    slots = np.concatenate([b * cap + np.arange(n) for b in range(batch)])
    gx = gpu(x)
    q = pk.rotate_rows(cfg, cache, gx[:, :8], gx[:, 8:10], gx[:, 10:], ints(np.tile(np.arange(n), batch)), ints(slots))
    assert torch.equal(q, gx[:, :8])
    dense = pk.sink_window_attend(cfg, q.view(batch, n, 8, D).transpose(1, 2).contiguous(), cache.K, cache.V, 0, 0, n, SCALE)
    paged = pk.paged_attend(cfg, q, cache, ints(np.arange(batch)[:, None]), ints([n] * batch), ints(np.arange(batch + 1) * n), SCALE,
                            max_tokens=n).view(batch, n, 8, D).transpose(1, 2)
    for b in range(batch):
        for h in range(8):
            k, v = (x[b * n:(b + 1) * n, c + h // g] for c in (8, 10))
            tol = tolerance(x[b * n:(b + 1) * n, h][:, None], k, v, SCALE)
            check(paged[b, h].cpu().numpy(), dense[b, h].double().cpu().numpy(), 2 * tol, f"seq {b} head {h}")
