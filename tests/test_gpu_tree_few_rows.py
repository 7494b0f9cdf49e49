"""Trees of few query rows per KV head, whose prefix goes through the kernels for chains, against 64 bits: at the numbers of rows where the way changes, with
segments joined in each of the ways there are, and with a workspace that calls of both ways share.  Bounds: see test_gpu_tree_attention."""
import pytest
import torch

import paper_2607_01831_b200 as lynx
from test_gpu_tree_attention import Problem, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,G", [(15, 1), (16, 1), (17, 1), (32, 1), (33, 1), (8, 2), (9, 2), (16, 2), (17, 2), (5, 3), (6, 5), (3, 5), (4, 8), (5, 8),
                                 (1, 16), (2, 16), (3, 16), (2, 12), (2, 11)])
@pytest.mark.parametrize("anchor", [False, True])
def test_where_the_way_changes(n, G, anchor):
    _check(Problem((1000, 17), n, 2, G, seed=n * G), anchor=anchor)
    _check(Problem((21000, 4000), n, 4, G, seed=n * G + 1), anchor=anchor)     # (several tiles a CTA)


@pytest.mark.parametrize("n,G", [(17, 1), (32, 1), (9, 2), (16, 2), (6, 3), (5, 4), (8, 4), (6, 5), (4, 7), (3, 8), (4, 8), (2, 11), (2, 16)])
@pytest.mark.parametrize("lens,Hkv", [((3000, 700), 4), ((0, 1, 129, 16), 2), ((200,) * 50, 1)])
def test_two_passes_over_the_anchor(n, G, lens, Hkv):
    """17 to 32 rows where the tables have room for 128 tiles per SM."""
    wide = 128 * 160 * 8 // (len(lens) * Hkv)
    pr = Problem(lens, n, Hkv, G, seed=n * G, extra_blocks=wide)
    _check(pr, anchor=True)
    _check(pr, anchor=True, out_f32=True)


@pytest.mark.parametrize("n,G", [(1, 4), (4, 4), (7, 4), (16, 1), (16, 2)])
@pytest.mark.parametrize("anchor", [False, True])
@pytest.mark.parametrize("lens,Hkv", [((32768,) + (64,) * 39, 1),      # one long segment among many
                                      ((500,) * 40 + (0, 3), 2),       # a slot or two
                                      ((100, 0, 7) * 20, 3),           # a unit at most
                                      ((9000,), 1), ((2000, 0), 2)])   # few segments
def test_ways_of_joining(n, G, anchor, lens, Hkv):
    _check(Problem(lens, n, Hkv, G, seed=n + Hkv), anchor=anchor)


@pytest.mark.parametrize("kind", ["tree", "chain", "random", "self", "none"])
@pytest.mark.parametrize("n,G", [(3, 4), (8, 4), (16, 2)])
@pytest.mark.parametrize("out_f32", [False, True])
def test_masks(kind, n, G, out_f32):
    _check(Problem((0, 40, 700), n, 1, G, kind=kind, seed=4), out_f32=out_f32)


@pytest.mark.parametrize("case", ["k_offset", "sharp", "flat_v", "big_v", "small_v", "uneven_v", "scale", "negative_scale"])
@pytest.mark.parametrize("n", [4, 8])
def test_values(case, n):
    kw = dict(k_offset=dict(k_off=20.0), sharp=dict(q_spread=12.0), flat_v=dict(v_rows=lambda z: torch.zeros_like(z)), big_v=dict(v_spread=1e30),
              small_v=dict(v_spread=1e-20), uneven_v=dict(v_rows=lambda z: torch.exp(3 * z))).get(case, {})
    pr = Problem((1500, 260), n, 2, 4, seed=21, **kw)
    _check(pr, scale=dict(scale=0.31, negative_scale=-0.05).get(case, 0.0))


def test_a_workspace_of_both_ways():
    """Full calls of 24 rows leave at zero what they find so, Anchor calls of as many and calls of 96 write beside it."""
    few, many = Problem((700, 300), 6, 2, 4, seed=5), Problem((3000, 800), 24, 2, 4, seed=6)
    d, e = few.device(), many.device()
    size = max(lynx.tree_workspace_bytes(p.geo, 2, p.n) for p in (few, many))
    d["workspace"] = e["workspace"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        _check(few, dev=d)
        _check(few, anchor=True, dev=d)
        _check(many, dev=e)
        _check(many, anchor=True, dev=e)


def test_streams_and_graphs():
    for n, anchor in ((4, False), (6, True), (7, False)):
        pr = Problem((900, 41), n, 2, 4, seed=n)
        d = pr.device()
        first = _check(pr, anchor=anchor, dev=d)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            other = lynx.tree_attention(**d, anchor_only=anchor)
        st.synchronize()
        assert torch.equal(first, other)
        out = torch.empty_like(first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lynx.tree_attention(**d, anchor_only=anchor, out=out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, out)


@pytest.mark.parametrize("n", [4, 8])
def test_bad_block_ids_are_reported(n):
    pr = Problem((100, 50), n, 1, 4, seed=61)
    d = pr.device()
    d["block_table"][1, 2] = 10 ** 6
    for p in (d["K"], d["V"]):
        p.meta.nan_to_num_(0.0, 0.0)
    lynx.tree_attention(**d)
    with pytest.raises(lynx.LynxError, match="block id"):
        lynx.check(d["workspace"])
    lynx.check(d["workspace"])
