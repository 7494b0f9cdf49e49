"""Outputs that the extension allocates are torch's own in every respect: a profiler lists them, and deterministic programs have them filled."""
import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu


def _recombine():
    planes = lynx.split_quantize(torch.randn(3, 2, 16, 128, device="cuda").to(torch.bfloat16))
    return lambda: lynx.recombine(planes)


def _plan():
    geo, pool = lynx.Geometry(8, 2, 16, 4, 4), lynx.make_block_pool(4, "cuda")
    table, lens = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    return lambda: lynx.plan_blocks(geo, pool, table, lens, lens, 8)


def _norm():
    q = torch.randn(5, 4, 128, device="cuda").to(torch.bfloat16)
    return lambda: lynx.norm_rotary(q, None)


@pytest.mark.parametrize("make", [_recombine, _plan, _norm])
@pytest.mark.parametrize("python", [False, True])
def test_allocations_are_seen_and_filled(make, python, monkeypatch):
    call = make()
    call()
    if python:
        for name in ("_fast_recombine", "_fast_plan_blocks", "_fast_norm_rotary"):
            monkeypatch.setattr(lynx, name, lynx._python_only)

    def seen():
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as p:
            out = call()
        torch.cuda.synchronize()
        return {e.key: e.count for e in p.key_averages()}, len([x for x in out if x is not None])

    ops, outputs = seen()
    assert ops.get("aten::empty", 0) + ops.get("aten::empty_like", 0) >= outputs and "aten::fill_" not in ops
    try:
        torch.use_deterministic_algorithms(True)
        ops, outputs = seen()
    finally:
        torch.use_deterministic_algorithms(False)
    assert ops.get("aten::fill_", 0) >= outputs
