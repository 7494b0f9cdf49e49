"""One workspace for calls of every batch and number of nodes up to those that it was made for, and for other tables: its size, and results that do not depend on what it
held."""
import random

import pytest
import torch

import paper_2607_01831_b200 as lynx
from test_gpu_tree_attention import Problem, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hkv", [1, 8])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 12, 16])
@pytest.mark.parametrize("blocks", [8, 24, 25, 300, 8192])
def test_the_size_never_falls(Hkv, G, blocks):
    geo = lynx.Geometry(Hkv * G, Hkv, 16, 64, blocks)
    batches, nodes = [1, 2, 3, 5, 8, 18, 19, 37, 64, 148, 300], list(range(1, 65))
    size = [[lynx.tree_workspace_bytes(geo, b, n) for n in nodes] for b in batches]
    assert min(map(min, size)) > 0
    assert all(x <= y for row in size for x, y in zip(row, row[1:]))
    assert all(x <= y for a, b in zip(size, size[1:]) for x, y in zip(a, b))


@pytest.mark.parametrize("G,Hkv", [(4, 2), (1, 3), (8, 1), (16, 1)])
def test_smaller_calls_and_other_tables(G, Hkv):
    """Calls of all sizes in turn, the largest again in between: each as with a workspace of its own."""
    shapes = [(3, 40), (3, 17), (3, 16), (2, 9), (1, 4), (3, 1), (1, 64 // G if G > 1 else 33)]
    shapes = [(b, min(n, 512 // G)) for b, n in shapes]
    lens = [(3000, 0, 700), (129, 1, 64), (260, 1500, 90)]
    cases = []
    for i, (b, n) in enumerate(shapes):
        # (tables as wide as the widest, and narrower ones)
        cases.append((Problem(lens[i % 3][:b], n, Hkv, G, seed=91 + i, extra_blocks=(0, 200, 40)[i % 3]), i % 2 == 1))
    devices = [pr.device() for pr, _ in cases]
    size = max(max(lynx.tree_workspace_bytes(pr.geo, 3, 40) for pr, _ in cases), max(d["workspace"].numel() for d in devices))
    shared = torch.zeros(size, dtype=torch.uint8, device="cuda")
    alone = [_check(pr, anchor=anchor, dev=d) for (pr, anchor), d in zip(cases, devices)]
    for d in devices:
        d["workspace"] = shared
    order = list(range(len(cases))) * 3
    random.Random(G).shuffle(order)
    for i in order:
        pr, anchor = cases[i]
        assert torch.equal(_check(pr, anchor=anchor, dev=devices[i]), alone[i])


@pytest.mark.parametrize("n,G", [(16, 4), (17, 4), (40, 2), (64, 8)])
def test_a_workspace_made_for_the_largest(n, G):
    """As an engine keeps it that drafts level by level: of each smaller call of the same tables, exactly the largest one's bytes are enough."""
    big = Problem((1200, 50), n, 2, G, seed=n)
    ws = lynx.make_tree_workspace(big.geo, 2, n, "cuda")
    for k in (1, 2, 3, 4, 5, 8, 9, 12, 15, 16, 17, 33, n):
        if k <= n:
            for anchor in (False, True):
                for b in (2, 1):
                    pr = Problem((1200, 50)[:b], k, 2, G, seed=k, extra_blocks=0)
                    pr.geo = lynx.Geometry(2 * G, 2, 16, pr.geo.num_blocks, big.geo.max_blocks_per_seq)
                    d = pr.device()
                    d["workspace"] = ws
                    _check(pr, anchor=anchor, dev=d)
