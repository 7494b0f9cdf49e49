"""The extension leaves the calls around the cache alone (returns None) where their arguments are no plain GPU tensors, and the Python
bodies then raise."""
import pytest
import torch

import paper_2607_01831_b200 as lynx

D = 128


def test_what_is_not_plain_is_left_alone():
    lynx.load()
    from paper_2607_01831_b200 import _native as n
    geo = lynx.Geometry(8, 2, 16, 4, 4)
    k, i = torch.zeros(3, 2, D, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32)
    planes, slots = lynx.alloc_planes((4, 2, 16), "cpu"), torch.zeros(3, dtype=torch.int64)
    spec = lynx.Rotary(torch.zeros(3, dtype=torch.int32), lynx.rotary_table(4))
    q = torch.zeros(1, 3, 8, D, dtype=torch.bfloat16)
    assert n.rotary(k, k, spec, None, None) is None and n.rotary(None, None, spec, None, None) is None and n.rotary(k) is None
    assert n.cache_append(geo, k, k, slots, planes, planes, None, None) is None and n.cache_append(object(), k, k, slots, planes, planes, None, spec) is None
    assert n.cache_read(geo, planes, planes, i, None, i[0, :2], 1, False, None, None) is None
    assert n.tree_attention(geo, q, planes, planes, i, i[0, :1], q[:, :, :2], q[:, :, :2], slots[None], slots, False, 0.0, None, None) is None
    with pytest.raises(lynx.LynxError, match="device tensors"):
        lynx.rotary(k, k, spec)
    with pytest.raises(lynx.LynxError, match="device tensors"):
        lynx.cache_append(geo, k, k, slots, planes, planes)
    with pytest.raises(lynx.LynxError, match="device tensors"):
        lynx.tree_attention(geo, q, planes, planes, i, i[0, :1], q[:, :, :2], q[:, :, :2], slots[None], slots)


def test_a_rotary_is_checked_when_it_is_made():
    pos, table = torch.zeros(2, 5, dtype=torch.int32), lynx.rotary_table(6, 16)
    assert lynx.Rotary(pos, table, [0, 1] * 8)._axis == bytes([0, 1] * 8) and lynx.Rotary(pos[0], table)._axis == bytes(16)
    for bad in ((pos.long(), table), (pos[None], table), (pos, table.double()), (pos, table[:, :31]), (pos, table, [0] * 15), (pos, table, [2] * 16),
                (pos, table, [-1] * 16), (pos, torch.zeros(3, 130))):
        with pytest.raises(lynx.LynxError):
            lynx.Rotary(*bad)
    with pytest.raises(Exception):
        lynx.Rotary(pos, table).positions = pos      # (what has been checked stays)
    want = torch.arange(6, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(16, dtype=torch.float64) / 16)
    assert torch.equal(table, torch.cat((want.cos(), want.sin()), 1).float())
