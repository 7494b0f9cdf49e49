"""An append whose source has no rows: every token is one whose source row is outside of it, and is left out."""
import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("python", [False, True])
@pytest.mark.parametrize("turned", [False, True])
def test_no_source_rows(python, turned, monkeypatch):
    H, bt, nb = 2, 16, 3
    geo = lynx.Geometry(H, H, bt, nb, nb)
    K, V = (lynx.Planes(torch.full((nb, H, bt, 64), 7, dtype=torch.uint8, device="cuda"), torch.full((nb, H, bt, 64), 7, dtype=torch.uint8, device="cuda"),
                        torch.full((nb, H, bt, 2), 7.0, device="cuda")) for _ in range(2))
    none = torch.empty(0, H, 128, dtype=torch.bfloat16, device="cuda")
    slots, rows = torch.arange(5, device="cuda"), torch.tensor([0, -1, 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    spec = lynx.Rotary(torch.empty(0, dtype=torch.int32, device="cuda"), lynx.rotary_table(4, device="cuda")) if turned else None
    if python:
        monkeypatch.setattr(lynx, "_fast_cache_append", lynx._python_only)
    lynx.cache_append(geo, none, none, slots, K, V, rows=rows, rotary=spec)
    lynx.cache_append(geo, none, none, slots[:0], K, V, rotary=spec)
    torch.cuda.synchronize()
    assert all((t == 7).all() for p in (K, V) for t in (p.anchor, p.residual, p.meta))
    with pytest.raises(lynx.LynxError):
        lynx.cache_append(geo, none, none, slots, K, V, rotary=spec)      # (without rows token i is row i)
