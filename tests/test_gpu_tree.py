"""GPU parity of the attention of drafted tokens over a cache (float16 and quantised) against float64."""

import numpy as np
import pytest
import torch

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE, attend64, check, draw, gpu, mask_words, random_tree, tolerance
from oracle import quant

pytestmark = pytest.mark.gpu


def _cfg(hkv, g):
    return pk.Config(hkv, g, 64, workloads.rotation_signs(3))


def _run(b, hkv, g, n, t, bits=None, mask="tree", lens=None, scale=SCALE, seed=0, law=1.0, cap=None):
    """One call checked in every output; rows of the cache past a sequence's length hold NaN."""
    print(f"[tree] batch {b} hkv {hkv} g {g} n {n} t {t} bits {bits} mask {mask} lens {lens}", flush=True)
    r = np.random.default_rng(seed)
    cfg = _cfg(hkv, g)
    cap = max(1, n) if cap is None else cap
    K, V = draw(r, b, hkv, cap, D, law=law), draw(r, b, hkv, cap, D)
    Kt, Vt, q = draw(r, b, hkv, t, D, law=law), draw(r, b, hkv, t, D), draw(r, b, hkv * g, t, D)
    size = [n] * b if lens is None else [min(max(x, 0), n) for x in lens]
    see = np.stack([np.tril(np.ones((t, t), bool)) if mask == "chain" else random_tree(r, t) for _ in range(b)])
    if mask == "holes":  # the last token sees nothing, the first is seen by nobody and holds NaN
        see[:, -1] = False
        see[:, :, 0] = False
        Kt[:, :, 0] = Vt[:, :, 0] = np.nan
    for s in range(b):
        K[s, :, size[s]:] = V[s, :, size[s]:] = np.nan
    words = None if mask == "chain" else gpu(mask_words(see))
    ln = None if lens is None else gpu(np.array(lens, np.int32))
    if bits:
        cache = pk.QuantCache.empty(cfg, b, cap, *bits)
        pk.quantize_rows(cfg, cache, gpu(np.nan_to_num(K)), gpu(np.nan_to_num(V)), 0, 0, cap)
        K, V = quant.round_trip(np.nan_to_num(K), bits[0]), quant.round_trip(np.nan_to_num(V), bits[1])
        out = pk.quant_tree_attend(cfg, gpu(q), cache, gpu(Kt), gpu(Vt), n, scale, mask=words, lens=ln)
    else:
        out = pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, scale, mask=words, lens=ln)
    out = out.cpu().numpy()
    for s in range(b):
        visible = np.concatenate([np.ones((t, size[s]), bool), see[s]], 1)
        for h in range(hkv * g):
            k_ = np.concatenate([K[s, h // g, :size[s]], Kt[s, h // g]]).astype(np.float64)
            v_ = np.concatenate([V[s, h // g, :size[s]], Vt[s, h // g]]).astype(np.float64)
            used = visible.any(0)
            k_, v_, vis = k_[used], v_[used], visible[:, used]
            want = attend64(q[s, h], k_, v_, vis, scale)
            check(out[s, h], want, tolerance(q[s, h], k_, v_, scale), f"seq {s} head {h}")
    return out


@pytest.mark.parametrize("g,t", [(1, 1), (4, 1), (16, 1), (3, 5), (4, 8), (2, 33), (7, 31), (4, 64), (16, 64), (1, 64)])
def test_rows_per_kv_head(g, t):
    _run(2, 2, g, 1000, t, seed=g * 100 + t)


@pytest.mark.parametrize("n", [0, 1, 15, 16, 31, 32, 33, 127, 128, 129, 255, 256, 257, 1023, 4097, 20001])
def test_lengths(n):
    _run(1, 2, 4, n, 4, seed=n)


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("g,n,t", [(4, 700, 1), (2, 33, 16), (4, 5000, 31), (8, 1, 8), (1, 0, 3)])
def test_quantised_cache(bits, g, n, t):
    _run(2, 2, g, n, t, bits=bits, seed=n + t)


@pytest.mark.parametrize("bits", [None, (8, 8), (4, 4)])
@pytest.mark.parametrize("t", [1, 6, 40])
def test_sequences_of_different_lengths(bits, t):
    # Lengths below 0 and above n are taken as 0 and n; the cache is larger than n.
    _run(5, 2, 4, 3000, t, bits=bits, lens=[0, 1, 3000, 1234, 2999], seed=t, cap=3100)
    _run(3, 1, 4, 500, t, bits=bits, lens=[-7, 501, 250], seed=t, cap=600)


@pytest.mark.parametrize("t", [2, 3, 33, 64])
@pytest.mark.parametrize("n", [0, 700])
def test_masks_with_empty_rows_and_unseen_drafts(n, t):
    out = _run(2, 2, 4, n, t, mask="holes", seed=t)
    if n == 0:
        assert not out[:, :, -1].any()


@pytest.mark.parametrize("bits", [None, (8, 8), (4, 4)])
@pytest.mark.parametrize("n", [100, 3000])  # one share of the keys, several
@pytest.mark.parametrize("g,t", [(1, 8), (4, 8), (4, 16), (4, 31), (2, 64)])
def test_drafts_that_are_not_finite_reach_only_tokens_that_see_them(g, t, n, bits):
    print(f"[tree] not finite: g {g} t {t} n {n} bits {bits}", flush=True)
    b, hkv = 2, 2
    r = np.random.default_rng(g + t + n)
    cfg = _cfg(hkv, g)
    K, V, q = draw(r, b, hkv, n, D), draw(r, b, hkv, n, D), draw(r, b, hkv * g, t, D)
    Kt, Vt = draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    see = np.stack([random_tree(r, t) for _ in range(b)])
    odd, lost = t // 2, t - 2  # a draft with such values, one whose score is NaN
    bad = Vt.copy()
    bad[:, :, odd, 3], bad[:, :, odd, 70], bad[:, :, odd, 127] = np.inf, -np.inf, np.nan
    bad[:, :, odd + 1, 3] = np.inf
    Vt[~np.isfinite(bad)] = 0
    badk = Kt.copy()
    badk[:, :, lost, 9] = np.nan
    Kt[:, :, lost] = 0
    mask = gpu(mask_words(see))
    if bits:
        cache = pk.QuantCache.empty(cfg, b, n, *bits)
        pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, n)
        K, V = quant.round_trip(K, bits[0]), quant.round_trip(V, bits[1])
        out = pk.quant_tree_attend(cfg, gpu(q), cache, gpu(badk), gpu(bad), n, SCALE, mask=mask).cpu().numpy()
    else:
        out = pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), gpu(badk), gpu(bad), n, SCALE, mask=mask).cpu().numpy()
    for s in range(b):
        dead, visible = see[s, :, lost], np.concatenate([np.ones((t, n), bool), see[s]], 1)
        for h in range(hkv * g):
            x, rows = out[s, h], bad[s, h // g].astype(np.float32)
            assert np.isnan(x[dead]).all()
            # Of the drafts that a token sees, the sum of such values of each dim (inf, -inf or NaN), else 0.
            odds = np.stack([np.where(np.isfinite(rows[m]), 0, rows[m]).sum(0) for m in see[s]])
            hit = (odds != 0) & ~dead[:, None]
            assert np.array_equal(x[hit], odds[hit], equal_nan=True)
            k_ = np.concatenate([K[s, h // g], Kt[s, h // g]]).astype(np.float64)
            v_ = np.concatenate([V[s, h // g], Vt[s, h // g]]).astype(np.float64)
            fine = ~hit & ~dead[:, None]
            want = attend64(q[s, h], k_, v_, visible)
            check(x[fine], want[fine], tolerance(q[s, h], k_, v_), f"seq {s} head {h}")


@pytest.mark.parametrize("t", [1, 32, 64])
def test_chain_without_a_mask(t):
    _run(2, 2, 3, 300, t, mask="chain", seed=t)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 1e-30])
def test_scales(scale):
    _run(1, 2, 4, 2000, 5, scale=scale, seed=3)


@pytest.mark.parametrize("groups", [(1, 1), (3, 3), (5, 7), (16, 4)])
def test_many_groups_and_shares(groups):
    _run(groups[0], groups[1], 2, 1500, 9, seed=5)


def test_scores_that_grow_along_the_cache():
    # Every step raises the running maximum; scores span hundreds of powers of two.
    b, hkv, g, n, t = 1, 1, 4, 4096, 4
    r = np.random.default_rng(8)
    q = np.abs(draw(r, b, hkv * g, t, D))
    K = (np.abs(draw(r, b, hkv, n, D)) * np.linspace(0.05, 6, n)[:, None]).astype(np.float16)
    V, Kt, Vt = draw(r, b, hkv, n, D), draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    for order in (slice(None), slice(None, None, -1)):
        Ko, Vo = K[:, :, order], V[:, :, order]
        out = pk.tree_attend(_cfg(hkv, g), gpu(q), gpu(Ko), gpu(Vo), gpu(Kt), gpu(Vt), n, SCALE).cpu().numpy()
        for h in range(g):
            k_, v_ = np.concatenate([Ko[0, 0], Kt[0, 0]]), np.concatenate([Vo[0, 0], Vt[0, 0]])
            vis = np.concatenate([np.ones((t, n), bool), np.tril(np.ones((t, t), bool))], 1)
            check(out[0, h], attend64(q[0, h], k_, v_, vis), tolerance(q[0, h], k_, v_), f"head {h}")


def test_equal_scores_average_the_values():
    b, hkv, g, n, t = 1, 1, 1, 9999, 1
    q = np.zeros((b, g, t, D), np.float16)
    r = np.random.default_rng(2)
    K, V = draw(r, b, hkv, n, D), draw(r, b, hkv, n, D)
    Kt, Vt = draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    out = pk.tree_attend(_cfg(1, 1), gpu(q), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, SCALE).cpu().numpy()
    want = np.concatenate([V[0, 0], Vt[0, 0]]).astype(np.float64).mean(0)
    # Float32 sums of 10000 values: at most 2^-24 a step of sums below sqrt(10000) 4.
    assert np.abs(out[0, 0, 0] - want).max() <= 1e4 * 2.0 ** -24 * 400 / 1e4


def test_the_quantised_cache_gives_what_its_values_give():
    # Over rows that the codes hold exactly, both caches hold the same values.
    b, hkv, g, n, t = 2, 2, 4, 777, 12
    r = np.random.default_rng(12)
    K, V = (quant.round_trip(draw(r, b, hkv, n, D), 8).astype(np.float16) for _ in range(2))
    Kt, Vt, q = draw(r, b, hkv, t, D), draw(r, b, hkv, t, D), draw(r, b, hkv * g, t, D)
    cfg = _cfg(hkv, g)
    cache = pk.QuantCache.empty(cfg, b, n)
    pk.quantize_rows(cfg, cache, gpu(K), gpu(V), 0, 0, n)
    x = pk.quant_tree_attend(cfg, gpu(q), cache, gpu(Kt), gpu(Vt), n, SCALE).cpu().numpy()
    y = pk.tree_attend(cfg, gpu(q), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, SCALE).cpu().numpy()
    for s in range(b):
        for h in range(hkv * g):
            check(x[s, h], y[s, h], 2 * tolerance(q[s, h], K[s, h // g], V[s, h // g]), f"seq {s} head {h}")


def test_a_long_cache_passes_32_bit_offsets():
    # One sequence, one head: 2^31 bytes and more of K behind the rows that are read (rows of 256 bytes).
    n, t = (1 << 23) + 1000, 2
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB")
    K = torch.zeros((1, 1, n, D), dtype=torch.float16, device="cuda")
    V = torch.zeros_like(K)
    r = np.random.default_rng(1)
    q = draw(r, 1, 2, t, D)
    at = n - 5
    K[0, 0, at] = gpu((8 * q[0, 0, 0].astype(np.float32)).astype(np.float16))
    V[0, 0, at] = 1
    Kt, Vt = torch.zeros((2, 1, 1, t, D), dtype=torch.float16, device="cuda")
    out = pk.tree_attend(_cfg(1, 2), gpu(q), K, V, Kt, Vt, n, SCALE).cpu().numpy()
    score = SCALE * 8 * (q[0, 0, 0].astype(np.float64) ** 2).sum()
    want = np.exp(score) / (np.exp(score) + n - 1 + 1)
    assert abs(out[0, 0, 0, 0] - want) <= 2 * (4 * np.sqrt(128) * 2.0 ** -24 * score + 2.0 ** -20)


def test_a_long_quantised_cache_passes_32_bit_offsets():
    # 127 million records of 272 bytes: records, their 16-byte pieces and bytes all pass 2^31.
    n, t = 127_000_000, 2
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    cfg = _cfg(1, 2)
    cache = pk.QuantCache.empty(cfg, 1, n)
    cache.rec.zero_()
    r = np.random.default_rng(1)
    q = draw(r, 1, 2, t, D)
    k, v = np.zeros((1, 1, 1, D), np.float16), np.ones((1, 1, 1, D), np.float16)
    k[0, 0, 0] = quant.round_trip((4 * q[0, 0, 0].astype(np.float32)).astype(np.float16), 8)
    pk.quantize_rows(cfg, cache, gpu(k), gpu(v), 0, n - 3, 1)
    Kt, Vt = torch.zeros((2, 1, 1, t, D), dtype=torch.float16, device="cuda")
    for scale in (SCALE, 4 * SCALE):  # two kernels' worth of rows: 2 heads x 2 drafts, and 33 rows below
        out = pk.quant_tree_attend(cfg, gpu(q), cache, Kt, Vt, n, scale).cpu().numpy()
        score = scale * (k[0, 0, 0].astype(np.float64) * q[0, 0, 0]).sum()
        want = np.exp(score) / (np.exp(score) + n - 1 + 1)
        assert abs(out[0, 0, 0, 0] - want) <= 2 * (4 * np.sqrt(128) * 2.0 ** -24 * score + 2.0 ** -20) + n * 2.0 ** -33
    cfg33 = _cfg(1, 3)
    q33 = np.repeat(q[:, :1, :1], 33, axis=1).reshape(1, 3, 11, D)
    Kt, Vt = torch.zeros((2, 1, 1, 11, D), dtype=torch.float16, device="cuda")
    out = pk.quant_tree_attend(cfg33, gpu(q33), cache, Kt, Vt, n, 4 * SCALE).cpu().numpy()
    assert np.abs(out[0, :, 0, 0] - want).max() <= 2 * (4 * np.sqrt(128) * 2.0 ** -24 * score + 2.0 ** -20) + n * 2.0 ** -33


def test_mask_bits_past_the_drafts_are_ignored():
    # The last draft is seen by nobody and holds NaN; bits t .. 63 are set in every word.
    b, hkv, g, n, t = 1, 2, 4, 100, 5
    r = np.random.default_rng(4)
    q, K, V = draw(r, b, hkv * g, t, D), draw(r, b, hkv, n, D), draw(r, b, hkv, n, D)
    Kt, Vt = draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)
    Kt[:, :, -1] = Vt[:, :, -1] = np.nan
    see = random_tree(r, t)
    see[:, -1] = False
    words = mask_words(see) | np.int64(-1 << t)
    for g_ in (g, 16):
        qq = draw(r, b, hkv * g_, t, D)
        out = pk.tree_attend(_cfg(hkv, g_), gpu(qq), gpu(K), gpu(V), gpu(Kt), gpu(Vt), n, SCALE, mask=gpu(words[None])).cpu().numpy()
        for h in range(hkv * g_):
            k_, v_ = np.concatenate([K[0, h // g_], Kt[0, h // g_, :-1]]), np.concatenate([V[0, h // g_], Vt[0, h // g_, :-1]])
            vis = np.concatenate([np.ones((t, n), bool), see[:, :-1]], 1)
            check(out[0, h], attend64(qq[0, h], k_, v_, vis), tolerance(qq[0, h], k_, v_), f"head {h}")


def test_two_streams_and_their_own_workspaces():
    b, hkv, g, n, t = 2, 2, 4, 3000, 8
    r = np.random.default_rng(6)
    cfg = _cfg(hkv, g)
    args = []
    for _ in range(2):
        args.append([gpu(x) for x in (draw(r, b, hkv * g, t, D), draw(r, b, hkv, n, D), draw(r, b, hkv, n, D),
                                      draw(r, b, hkv, t, D), draw(r, b, hkv, t, D))])
    alone = [pk.tree_attend(cfg, *a, n, SCALE) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        outs = [pk.tree_attend(cfg, *a, n, SCALE, stream=s) for a, s in zip(args, streams)]
        torch.cuda.synchronize()
        for x, y in zip(alone, outs):
            assert torch.equal(x, y)


def test_captured_calls_replay():
    b, hkv, g, n, t = 3, 2, 4, 2000, 8
    r = np.random.default_rng(9)
    cfg = _cfg(hkv, g)
    q, K, V, Kt, Vt = (gpu(x) for x in (draw(r, b, hkv * g, t, D), draw(r, b, hkv, n, D), draw(r, b, hkv, n, D),
                                        draw(r, b, hkv, t, D), draw(r, b, hkv, t, D)))
    lens = torch.zeros(b, dtype=torch.int32, device="cuda")
    mask = torch.zeros((b, t), dtype=torch.int64, device="cuda")
    out = torch.zeros_like(q, dtype=torch.float32)
    ws = torch.empty(pk.tree_workspace_size(cfg, b, n, t), dtype=torch.uint8, device="cuda")

    def call():
        pk.tree_attend(cfg, q, K, V, Kt, Vt, n, SCALE, mask=mask, lens=lens, out=out, workspace=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        lens.copy_(gpu(r.integers(0, n + 1, b).astype(np.int32)))
        mask.copy_(gpu(np.stack([mask_words(random_tree(r, t)) for _ in range(b)])))
        q.copy_(gpu(draw(r, b, hkv * g, t, D)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
