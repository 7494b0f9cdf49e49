"""Trees whose rows have little to do with one another: sequences with fewer nodes than the call, whose other rows may hold anything, and rows of very
different magnitudes.  Every other row's result is what it is without them, within the bounds of test_gpu_tree_attention (E is a row's own: 2^-16 of the
largest sum of magnitudes that enters one of its scores)."""
import math

import pytest
import torch

import paper_2607_01831_b200 as lynx
from test_gpu_tree_attention import NAN, Problem

pytestmark = pytest.mark.gpu

INF = float("inf")
GARBAGE = [INF, -INF, NAN, 1e30, 3e38, -1e5, 2.0 ** 24]     # of queries
# (nodes, heads, Anchor) whose prefix goes through the kernels for chains: up to 16 rows, 32 on the full codes
FEW = [(4, 1, False), (4, 4, False), (7, 2, False), (16, 1, False), (8, 4, False), (5, 5, False), (2, 16, False), (10, 3, False),
       (4, 1, True), (4, 4, True), (7, 2, True), (16, 1, True), (2, 8, True), (3, 5, True)]
# through tree_attention_kernel: up to 32 rows (four lanes of tensor memory each), 64 (two), 128, and row blocks
MANY = [(31, 1, False), (8, 4, True), (5, 5, True), (9, 4, False), (16, 4, True), (32, 2, False), (17, 4, False), (32, 4, True), (32, 4, False), (40, 4, False),
        (64, 8, True)]


def _pad(pr, real):
    """Leaves the first real[b] nodes of each sequence: the rest sees nothing and is seen by none, and its keys and values are NaN."""
    live = torch.zeros(pr.B, pr.n, dtype=torch.bool)
    for b, n in enumerate(real):
        live[b, :n] = True
        pr.sees[b, n:], pr.sees[b, :, n:] = False, False
        pr.kn[b, n:], pr.vn[b, n:] = NAN, NAN
    return live


def _call(pr, anchor, scale=0.0, out_f32=True):
    d = pr.device()
    lse = torch.full(pr.q.shape[:3], 777.0, device="cuda")
    out = torch.empty(pr.q.shape, dtype=torch.float32 if out_f32 else torch.bfloat16, device="cuda")
    lynx.tree_attention(**d, anchor_only=anchor, softmax_scale=scale, lse=lse, out=out)
    lynx.check(d["workspace"])
    return out, lse


def _compare(rows, got, lse, want, out_f32=True):
    """rows: bool [B][n][Hq] or [B][n], those that are compared; want: what Problem.exact() gives."""
    out, want_lse, A, E = want
    rows = rows.cuda() if rows.dim() == 3 else rows.cuda()[..., None].expand(want_lse.shape)
    tol = ((2.0 ** -9 + 2 * E) * A)[..., None] + (0.0 if out_f32 else 2.0 ** -8) * out.abs() + 1e-30
    err = (got.double() - out).abs()
    assert torch.isfinite(got[rows]).all()
    assert (err <= tol)[rows].all(), (err / tol)[rows].max().item()
    empty = want_lse == -math.inf
    assert torch.equal((lse == -math.inf)[rows], empty[rows]) and (got[rows & empty] == 0).all()
    full = rows & ~empty
    off = (lse.double() - want_lse).abs()
    assert (off <= E + 2.0 ** -18 * (1 + want_lse.abs()))[full].all(), off[full].max().item()


def _padding(lens, real, n, G, Hkv, anchor, seed, extra_blocks=0, kind="tree"):
    pr = Problem(lens, n, Hkv, G, seed=seed, extra_blocks=extra_blocks, kind=kind)
    live = _pad(pr, real)
    assert not live.all() and live.any()
    pads = [(b, j) for b in range(pr.B) for j in range(n) if not live[b, j]]
    g = torch.Generator().manual_seed(seed)
    clean = pr.q.clone()
    for i, (b, j) in enumerate(pads):
        x = GARBAGE[i % len(GARBAGE)]
        some = torch.rand(pr.q.shape[2:], generator=g) < (1.0 if i % 2 else 0.3)
        clean[b, j] = 0.0
        pr.q[b, j][some] = x
    for x in (pads[0], pads[-1]):          # (each of a call's pads is large)
        pr.q[x][:, 5] = 1e30
    garbage, pr.q = pr.q, clean
    want = pr.exact(anchor)
    pr.q = garbage
    got, lse = _call(pr, anchor)
    _compare(live, got, lse, want)


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
def test_what_padding_holds(n, G, anchor):
    _padding((700, 40, 300), (max(1, n // 2), max(1, n - 1), 1), n, G, 2, anchor, seed=n + G)
    _padding((9000,), (n - 1,), n, G, 1, anchor, seed=n + G + 1)


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
def test_what_padding_holds_where_no_row_sees_a_node(n, G, anchor):
    """The rows that are meant attend to the prefix alone, as the padding does: nothing tells them apart."""
    _padding((700, 40, 300), (max(1, n // 2), max(1, n - 1), 1), n, G, 2, anchor, seed=n + G, kind="none")
    _padding((5000,), (1,), n, G, 1, anchor, seed=n + G + 1, kind="none")


@pytest.mark.parametrize("n,G", [(17, 1), (8, 4), (4, 8), (6, 5)])
def test_what_padding_holds_in_two_passes(n, G):
    _padding((300, 40), (max(1, n // 3), n - 1), n, G, 4, True, seed=n, extra_blocks=128 * 160)


def _magnitudes(n, G, anchor, lens, seed):
    """Rows without nodes whose queries are 2^20 times the others'; scores of ordinary size in the others, then in them."""
    pr = Problem(lens, n, 2, G, seed=seed, kind="self")
    pr.sees[:, 1::2, 1::2] = False             # every other row sees no node
    pr.kn[:, 1::2], pr.vn[:, 1::2] = NAN, NAN
    with_nodes = pr.sees.any(2)
    pr.q[with_nodes] = (pr.q[with_nodes].float() * 2.0 ** -20).to(torch.bfloat16)
    for rows, scale in ((with_nodes, 2.0 ** 20 / 128 ** 0.5), (torch.ones_like(with_nodes), 1 / 128 ** 0.5)):
        want = pr.exact(anchor, scale)
        for out_f32 in (True, False):
            got, lse = _call(pr, anchor, scale, out_f32)
            assert torch.isfinite(got).all()   # (too large a score has no bound, but a row)
            _compare(rows, got, lse, want, out_f32)


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
def test_larger_rows_without_nodes(n, G, anchor):
    _magnitudes(n, G, anchor, (500, 30), seed=n * G)
    _magnitudes(n, G, anchor, (6000,), seed=n * G + 1)


def _no_number(n, G, anchor, lens, seed):
    """A row with an infinity or a NaN in its query, although it sees nodes: the others are what they are."""
    pr = Problem(lens, n, 2, G, seed=seed, kind="chain")
    want = pr.exact(anchor)
    for x in (INF, NAN):
        pr.q[0, n // 2, G - 1, 7], pr.q[-1, 0, 0, 100] = x, x
        rows = torch.isfinite(pr.q.float()).all(-1)
        got, lse = _call(pr, anchor)
        _compare(rows, got, lse, want)


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
def test_a_row_that_is_no_number(n, G, anchor):
    _no_number(n, G, anchor, (700, 33), seed=n + G)


def _strange_node(n, G, anchor, lens, seed, kind):
    """A node whose key or value holds what is no number, or the largest there is: rows that do not see it are what they are without it, and where a value is no
    number, neither are the results of the rows that see it."""
    for i, (key, value) in enumerate([(INF, None), (NAN, None), (3e38, None), (None, INF), (None, NAN), (-INF, NAN)]):
        pr = Problem(lens, n, 2, G, seed=seed + i, kind=kind)
        node = (i * 7 + n // 2) % n
        pr.kn[:, node], pr.vn[:, node] = 0.0, 0.0       # (in what is compared with)
        want = pr.exact(anchor)
        pr.kn[:, node], pr.vn[:, node] = 0.5, 0.5
        if key is not None:
            pr.kn[:, node, :, 3::17] = key
        if value is not None:
            pr.vn[:, node, :, 100] = value
        sees = pr.sees[:, :, node]
        for out_f32 in (True, False):
            got, lse = _call(pr, anchor, out_f32=out_f32)
            _compare(~sees, got, lse, want, out_f32)
            if value is not None and sees.any():
                assert not torch.isfinite(got[sees.cuda()][..., 100]).any()


def _no_lse(n, G, anchor, seed):
    """The log-sum-exp of a row that sees a node with a NaN in its key is none, nor is it that of an empty row."""
    pr = Problem((150, 0, 33), n, 2, G, seed=seed, kind="tree")
    pr.kn[:, n // 2, :, 9] = NAN
    sees = pr.sees[:, :, n // 2].cuda()
    got, lse = _call(pr, anchor)
    assert torch.isnan(got[sees]).all() and torch.isnan(lse[sees]).all() and torch.isfinite(lse[~sees]).all()


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
@pytest.mark.parametrize("kind", ["self", "tree"])
def test_a_node_that_is_no_number(n, G, anchor, kind):
    _strange_node(n, G, anchor, (150, 0, 33), n * G, kind)


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
def test_no_log_sum_exp_of_what_is_no_number(n, G, anchor):
    _no_lse(n, G, anchor, seed=n + G)


def _strange_prefix(n, G, anchor, lens, seed):
    """A token of the prefix whose scale is infinite, as of a row that was quantised with an infinity in it: all rows of its sequence see it and are no numbers, the
    other sequences' are what they are."""
    for tensor in (0, 1):
        pr = Problem(lens, n, 2, G, seed=seed + tensor, kind="tree")
        want = pr.exact(anchor)
        token = lens[0] // 2
        pr.planes[tensor][2][pr.table[0, token // 16], :, token % 16] = torch.tensor([INF, 1.0])
        got, lse = _call(pr, anchor)
        assert not torch.isfinite(got[0]).any()
        assert tensor == 1 or not torch.isfinite(lse[0]).any() and not (lse[0] == -INF).any()
        rows = torch.ones(pr.B, n, dtype=torch.bool)
        rows[0] = False
        _compare(rows, got, lse, want)


@pytest.mark.parametrize("n,G,anchor", FEW + MANY)
def test_a_prefix_that_is_no_number(n, G, anchor):
    _strange_prefix(n, G, anchor, (40, 90, 0), seed=n + G)
    _strange_prefix(n, G, anchor, (7000, 300), seed=n + G)
    _strange_prefix(n, G, anchor, (300,) * 50, seed=n + G)
    _strange_prefix(n, G, anchor, (32768,) + (64,) * 39, seed=n + G)     # (joined by each of the ways there are)
