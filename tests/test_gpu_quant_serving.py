"""The quantised cache and the several-token calls together, as a serving program uses them: a padded prompt, its rows
into the index and the cache, decode steps over retrieved rows and the window, drafts verified and the accepted ones
written; every call against float64 over the values that the cache stands for."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, attend64, check, draw, gpu, mask_words, random_tree, tolerance
from oracle import quant

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kb,vb,host", [(8, 8, False), (8, 4, True), (4, 4, False)])
def test_prompt_decode_and_drafts(kb, vb, host):
    b, hkv, g, t0, cap = 2, 2, 4, 700, 760
    r = np.random.default_rng(kb + vb)
    cfg = pk.Config(hkv, g, cap, workloads.rotation_signs(5))
    lens = np.array([700, 633])  # the second prompt is padded
    K, V = draw(r, b, hkv, cap, D), draw(r, b, hkv, cap, D)
    Kd, Vd = gpu(K), gpu(V)

    # The prompt, in a chunk of 512 and the rest, over sinks and a window.
    q = draw(r, b, hkv * g, t0, D)
    out = torch.zeros((b, hkv * g, t0, D), dtype=torch.float16, device="cuda")
    for pos, t in ((0, 512), (512, t0 - 512)):
        part = torch.zeros((b, hkv * g, t, D), dtype=torch.float16, device="cuda")
        counts = gpu(np.clip(lens - pos, 0, t).astype(np.int32))
        pk.sink_window_attend(cfg, gpu(q[:, :, pos:pos + t]), Kd, Vd, pos, 16, 256, SCALE, counts=counts, out=part)
        out[:, :, pos:pos + t] = part
    out = out.cpu().numpy()
    for s in range(b):
        p, j = np.arange(lens[s])[:, None], np.arange(lens[s])[None]
        vis = (j <= p) & ((j < 16) | (j > p - 256))
        for h in range(hkv * g):
            k_, v_, q_ = K[s, h // g, :lens[s]], V[s, h // g, :lens[s]], q[s, h, :lens[s]]
            check(out[s, h, :lens[s]], attend64(q_, k_, v_, vis), tolerance(q_, k_, v_, half_out=True), f"prompt {s} {h}")
        assert not out[s, :, lens[s]:].any()

    # Its rows into the index and the cache.
    cache = pk.QuantCache.empty(cfg, b, cap, kb, vb, host_mapped=host)
    cache.rec.zero_()
    pk.quantize_rows(cfg, cache, Kd, Vd, 0, 0, t0)
    index = pk.Index.empty(cfg, b)
    n = 600  # rows of the Retrieval region behind 16 sinks; Local is what follows
    pk.encode(cfg, index, Kd[:, :, 16:16 + n].contiguous())
    Kh, Vh = quant.round_trip(K[:, :, :t0], kb), quant.round_trip(V[:, :, :t0], vb)

    # A decode step: retrieval, then attention over the winners alone, and with the window.
    q1 = draw(r, b, hkv * g, D)
    budget = pk.Budget(128, 256, 32)
    idx, _, _ = pk.retrieve(cfg, index, gpu(q1), n, budget)
    o1 = pk.quant_attend(cfg, gpu(q1), cache, idx + 16, SCALE).cpu().numpy()
    win = pk.Window(16, 16, 16 + n, 633)
    wcap = 16 + 40
    Kw, Vw = np.zeros((2, b, hkv, wcap, D), np.float16)
    dense = list(range(16)) + list(range(16 + n, 633))
    for row in dense:
        Kw[:, :, pk.window_slot(row, 16, wcap)] = K[:, :, row]
        Vw[:, :, pk.window_slot(row, 16, wcap)] = V[:, :, row]
    o2 = pk.quant_tiered_attend(cfg, gpu(q1), gpu(Kw), gpu(Vw), cache, idx, win, SCALE).cpu().numpy()
    rows = idx.cpu().numpy()
    for s in range(b):
        for h in range(hkv * g):
            at = rows[s, h] + 16
            k_, v_ = Kh[s, h // g, at], Vh[s, h // g, at]
            check(o1[s, h][None], attend64(q1[s, h][None], k_, v_, np.ones((1, 32), bool)),
                  tolerance(q1[s, h][None], k_, v_), f"winners {s} {h}")
            k_ = np.concatenate([K[s, h // g, dense].astype(np.float64), k_])
            v_ = np.concatenate([V[s, h // g, dense].astype(np.float64), v_])
            check(o2[s, h][None], attend64(q1[s, h][None], k_, v_, np.ones((1, len(k_)), bool)),
                  tolerance(q1[s, h][None], k_, v_), f"window {s} {h}")

    # Drafts over every cached row; the first three of a chain are accepted and written behind each sequence.
    if host:
        device = pk.QuantCache(cache.rec.cuda(), kb, vb)
    else:
        device = cache
    t = 11
    see = np.stack([random_tree(r, t) for _ in range(b)])
    qt, Kt, Vt = draw(r, b, hkv * g, t, D), draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    ln = gpu(lens.astype(np.int32))
    o3 = pk.quant_tree_attend(cfg, gpu(qt), device, gpu(Kt), gpu(Vt), t0, SCALE, mask=gpu(mask_words(see)),
                              lens=ln).cpu().numpy()
    pk.quantize_rows(cfg, device, gpu(Kt), gpu(Vt), 0, ln, 3)
    q4, K4, V4 = draw(r, b, hkv * g, 1, D), draw(r, b, hkv, 1, D), draw(r, b, hkv, 1, D)
    o4 = pk.quant_tree_attend(cfg, gpu(q4), device, gpu(K4), gpu(V4), t0 + 3, SCALE, lens=ln + 3).cpu().numpy()
    Ka, Va = quant.round_trip(Kt[:, :, :3], kb), quant.round_trip(Vt[:, :, :3], vb)
    for s in range(b):
        m = lens[s]
        for h in range(hkv * g):
            k_ = np.concatenate([Kh[s, h // g, :m], Kt[s, h // g].astype(np.float64)])
            v_ = np.concatenate([Vh[s, h // g, :m], Vt[s, h // g].astype(np.float64)])
            vis = np.concatenate([np.ones((t, m), bool), see[s]], 1)
            check(o3[s, h], attend64(qt[s, h], k_, v_, vis), tolerance(qt[s, h], k_, v_), f"drafts {s} {h}")
            k_ = np.concatenate([Kh[s, h // g, :m], Ka[s, h // g], K4[s, h // g].astype(np.float64)])
            v_ = np.concatenate([Vh[s, h // g, :m], Va[s, h // g], V4[s, h // g].astype(np.float64)])
            check(o4[s, h], attend64(q4[s, h], k_, v_, np.ones((1, m + 4), bool)), tolerance(q4[s, h], k_, v_), f"next {s} {h}")


def test_a_captured_decode_step_advances_by_its_device_positions():
    # Write, index-free attention over the whole cache and the next position, all in one graph.
    b, hkv, g, cap = 2, 2, 2, 300
    r = np.random.default_rng(2)
    cfg = pk.Config(hkv, g, cap, workloads.rotation_signs(5))
    cache = pk.QuantCache.empty(cfg, b, cap)
    cache.rec.zero_()
    n0 = np.array([250, 17], np.int32)
    K0, V0 = draw(r, b, hkv, cap, D), draw(r, b, hkv, cap, D)
    pk.quantize_rows(cfg, cache, gpu(K0), gpu(V0), 0, 0, cap)
    lens = gpu(n0)
    q, K1, V1 = (torch.zeros((b, h, 1, D), dtype=torch.float16, device="cuda") for h in (hkv * g, hkv, hkv))
    out = torch.zeros((b, hkv * g, 1, D), device="cuda")
    ws = torch.empty(pk.tree_workspace_size(cfg, b, cap, 1), dtype=torch.uint8, device="cuda")

    def step():
        pk.quant_tree_attend(cfg, q, cache, K1, V1, cap, SCALE, lens=lens, out=out, workspace=ws)
        pk.quantize_rows(cfg, cache, K1, V1, 0, lens, 1)
        lens.add_(1)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lens.copy_(gpu(n0))
    Kh, Vh = quant.round_trip(K0, 8), quant.round_trip(V0, 8)
    pk.quantize_rows(cfg, cache, gpu(K0), gpu(V0), 0, 0, cap)
    n = n0.copy()
    for _ in range(5):
        fresh = draw(r, b, hkv * g, 1, D), draw(r, b, hkv, 1, D), draw(r, b, hkv, 1, D)
        for x, y in zip((q, K1, V1), fresh):
            x.copy_(gpu(y))
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        for s in range(b):
            for h in range(hkv * g):
                k_ = np.concatenate([Kh[s, h // g, :n[s]], fresh[1][s, h // g].astype(np.float64)])
                v_ = np.concatenate([Vh[s, h // g, :n[s]], fresh[2][s, h // g].astype(np.float64)])
                check(got[s, h], attend64(fresh[0][s, h], k_, v_, np.ones((1, n[s] + 1), bool)),
                      tolerance(fresh[0][s, h], k_, v_), f"step {n} {s} {h}")
            Kh[s, :, n[s]] = quant.round_trip(fresh[1][s, :, 0], 8)
            Vh[s, :, n[s]] = quant.round_trip(fresh[2][s, :, 0], 8)
        n += 1
        assert (lens.cpu().numpy() == n).all()
