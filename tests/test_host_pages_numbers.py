"""Whole numbers past the C types of the paged cache's entry points: refused or taken as the largest, never wrapped.
Nothing is launched: no GPU needed."""

import os

import pytest
import torch

import paper_2602_07721_amd as pk
import workloads

pytestmark = pytest.mark.skipif(not os.path.exists(pk.LIB_PATH), reason="library not built")

i32 = torch.int32


def _cfg():
    return pk.Config(2, 4, 1, workloads.rotation_signs(3))


def test_workspace_sizes():
    cfg = _cfg()
    assert pk.paged_workspace_size(cfg, 2 ** 32 + 1, 4, 1) == pk.paged_workspace_size(cfg, 1, 2 ** 64 + 4, 1) == 0
    assert pk.paged_workspace_size(cfg, 1 - 2 ** 32, 4, 1) == pk.paged_workspace_size(cfg, 1, 4, 1 - 2 ** 64) == 0
    assert pk.paged_workspace_size(cfg, 3, 400, 2 ** 64 + 1) == pk.paged_workspace_size(cfg, 3, 400, 400)


@pytest.mark.parametrize("size", [2 ** 32 + 16, 16 - 2 ** 32, 2 ** 40])
def test_page_sizes(monkeypatch, size):
    monkeypatch.setattr(pk, "_require_on", lambda *a: None)  # tensors of the CPU: refused before any launch
    monkeypatch.setattr(pk, "_stream", lambda s: None)
    with pytest.raises(pk.PariskvError) as e:
        pk.plan_pages(torch.zeros(2, 8, dtype=i32), torch.zeros(10, dtype=i32), torch.zeros(1, dtype=i32),
                      torch.zeros(2, dtype=i32), torch.zeros(2, dtype=i32), size, plan=pk.PagePlan.empty(2, 5, device="cpu"))
    assert e.value.code == pk.ERR_INVALID


def test_most_tokens(monkeypatch):
    # What reaches the library: the largest number, not 1.
    seen = []
    monkeypatch.setattr(pk, "_require_on", lambda *a: None)
    monkeypatch.setattr(pk, "_stream", lambda s: None)
    monkeypatch.setattr(pk.lib(), "pariskv_paged_attend", lambda *a: seen.append(a) or pk.OK)
    half = torch.float16
    cache = pk.PagedCache(torch.zeros(10, 2, 16, 128, dtype=half), torch.zeros(10, 2, 16, 128, dtype=half))
    pk.paged_attend(_cfg(), torch.zeros(4, 8, 128, dtype=half), cache, torch.zeros(3, 8, dtype=i32), torch.zeros(3, dtype=i32),
                    torch.zeros(4, dtype=i32), 0.1, max_tokens=2 ** 64 + 1, out=torch.zeros(4, 8, 128, dtype=half),
                    workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    assert 2 ** 63 - 1 in seen[0]
