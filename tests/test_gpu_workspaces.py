"""One workspace, sized for the largest call, through a generation's shorter ones."""

import pytest
import torch

import paper_2602_07721_amd as pk
import workloads
from new_tokens import D, SCALE

pytestmark = pytest.mark.gpu


def _randn(*shape):
    return torch.randn(*shape, device="cuda").half()


@pytest.mark.parametrize("bits", [None, (8, 8)])
def test_drafts(bits):
    b, hkv, g, n, t = 3, 2, 4, 16448, 8
    cfg = pk.Config(hkv, g, 64, workloads.rotation_signs(3))
    torch.manual_seed(1)
    K, V = _randn(b, hkv, n, D), _randn(b, hkv, n, D)
    ws = torch.empty(pk.tree_workspace_size(cfg, b, n, t), dtype=torch.uint8, device="cuda")
    for b_, n_, t_ in ((3, 16448, 8), (3, 16384, 8), (1, 16320, 8), (2, 100, 3), (1, 5000, 1), (3, 0, 2)):
        print(f"[workspace] drafts batch {b_} n {n_} t {t_} bits {bits}", flush=True)
        Kb, Vb = K[:b_].contiguous(), V[:b_].contiguous()
        q, Kt, Vt = _randn(b_, hkv * g, t_, D), _randn(b_, hkv, t_, D), _randn(b_, hkv, t_, D)
        if bits:
            cache = pk.QuantCache.empty(cfg, b_, n, *bits)
            pk.quantize_rows(cfg, cache, Kb, Vb, 0, 0, n)
            x, y = (pk.quant_tree_attend(cfg, q, cache, Kt, Vt, n_, SCALE, workspace=w) for w in (ws, None))
        else:
            x, y = (pk.tree_attend(cfg, q, Kb, Vb, Kt, Vt, n_, SCALE, workspace=w) for w in (ws, None))
        assert torch.equal(x, y)


def test_windows():
    b, hkv, g, pos, t = 2, 2, 4, 6000, 1200
    cfg = pk.Config(hkv, g, 64, workloads.rotation_signs(3))
    torch.manual_seed(2)
    K, V = _randn(b, hkv, pos + t, D), _randn(b, hkv, pos + t, D)
    ws = torch.empty(pk.sink_window_workspace_size(cfg, b, pos, t, 64, 4096), dtype=torch.uint8, device="cuda")
    for b_, pos_, t_ in ((2, 0, 1200), (2, 6000, 1200), (2, 6000, 1), (1, 5000, 40), (1, 4096, 480), (2, 6000, 16)):
        print(f"[workspace] window batch {b_} pos {pos_} t {t_}", flush=True)
        Kb, Vb, q = K[:b_].contiguous(), V[:b_].contiguous(), _randn(b_, hkv * g, t_, D)
        x, y = (pk.sink_window_attend(cfg, q, Kb, Vb, pos_, 64, 4096, SCALE, workspace=w) for w in (ws, None))
        assert torch.equal(x, y)
