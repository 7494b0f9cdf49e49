"""Attention of a tree of drafted tokens over the planes, against a plain evaluation in 64 bits.

Bounds.  Weights and values enter the second product as FP16: a weight is off by 2^-11 of itself at most, a value
mid + scale (c - 128) by 2^-11 of each of its factors' and its own magnitude, 2^-9 of A in all, A = sum_t w_t (|mid_t| + 128 |scale_t|) over a
row's weights w (nodes: their largest |v|).  Scores: keys' deviations from the middle of their row enter exactly, middles in two FP16
parts (2^-22); FP32 sums over 128 channels of them and of mid x sum(q), and the factors of a row, are off by E = 2^-16 of S at most, S the
largest sum of magnitudes that enters one.  A weight follows relatively and the
output by twice that of A.  The last rounding to BF16 is 2^-8 of the output; log-sum-exps are off by the scores' error, the sum's
rounding and the approximations of exp2 and log2 (2^-18)."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2607_01831_b200 as lynx
from util import bf16_bits

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _nibbles(t):
    return torch.stack((t & 15, t >> 4), -1).flatten(-2).double()


def _tree_masks(B, n, kind, g):
    m = torch.zeros(B, n, n, dtype=torch.bool)
    for b in range(B):
        for j in range(n):
            if kind == "tree":
                if j:
                    m[b, j] = m[b, int(torch.randint(max(0, j - 5), j, (1,), generator=g))]
                m[b, j, j] = True
            elif kind == "chain":
                m[b, j, :j + 1] = True
            elif kind == "random":
                m[b, j] = torch.rand(n, generator=g) < 0.3
            elif kind == "self":
                m[b, j, j] = True
    return m


def _as_words(m):
    B, n, _ = m.shape
    words = [[sum(1 << i for i in range(n) if m[b, j, i]) for j in range(n)] for b in range(B)]
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in ws] for ws in words], dtype=torch.int64)


class Problem:
    def __init__(self, lens, n, Hkv, G, bt=16, kind="tree", seed=0, k_off=0.0, v_spread=1.0, q_spread=1.0, extra_blocks=0, v_rows=None):
        g = torch.Generator().manual_seed(seed)
        self.B, self.n, self.Hkv, self.G, self.bt, self.lens = len(lens), n, Hkv, G, bt, list(lens)
        B, Hq = self.B, Hkv * G
        need = [max(1, -(-x // bt)) for x in lens]
        nb = sum(need) + 2
        ids = torch.randperm(nb, generator=g).to(torch.int32)
        self.table = torch.zeros(B, max(need) + extra_blocks, dtype=torch.int32)
        for b, x in enumerate(need):
            self.table[b, :x] = ids[sum(need[:b]):sum(need[:b]) + x]
        self.geo = lynx.Geometry(Hq, Hkv, bt, nb, self.table.shape[1])
        k = torch.randn(nb, Hkv, bt, 128, generator=g) + k_off
        v = torch.randn(nb, Hkv, bt, 128, generator=g) * v_spread
        if v_rows is not None:
            v = v * v_rows(torch.randn(nb, Hkv, bt, 1, generator=g))
        self.planes = []
        for x in (k, v):
            a, r, m = oracle.split_quantize(bf16_bits(x.to(torch.bfloat16)))
            self.planes.append([torch.from_numpy(np.ascontiguousarray(t)).view(nb, Hkv, bt, -1) for t in (a, r, m)])
        # what lies behind a sequence's end, and in blocks of none, is anything
        live = torch.zeros(nb, bt, dtype=torch.bool)
        for b, x in enumerate(lens):
            t = torch.arange(x)
            live[self.table[b, t // bt].long(), t % bt] = True
        for p in self.planes:
            p[2][(~live)[:, None].expand(nb, Hkv, bt)] = torch.tensor([NAN, float("inf")])
            p[0][(~live)[:, None].expand(nb, Hkv, bt)] = 0xA5
        self.q = (torch.randn(B, n, Hq, 128, generator=g) * q_spread).to(torch.bfloat16)
        self.kn = (torch.randn(B, n, Hkv, 128, generator=g) + k_off).to(torch.bfloat16)
        self.vn = (torch.randn(B, n, Hkv, 128, generator=g) * v_spread).to(torch.bfloat16)
        self.sees = _tree_masks(B, n, kind, g)
        unused = ~self.sees.any(1)
        self.kn[unused], self.vn[unused] = NAN, NAN     # (nodes that no row sees)

    def device(self):
        K, V = (lynx.Planes(*(t.cuda() for t in p)) for p in self.planes)
        vn = torch.zeros(self.B, self.n, 3 * self.Hkv, 128, dtype=torch.bfloat16, device="cuda")
        vn[:, :, self.Hkv:2 * self.Hkv] = self.vn.cuda()
        return dict(geo=self.geo, q=self.q.cuda(), K=K, V=V, block_table=self.table.cuda(),
                    seq_lens=torch.tensor(self.lens, dtype=torch.int32).cuda(), k_nodes=self.kn.cuda(),
                    v_nodes=vn[:, :, self.Hkv:2 * self.Hkv], tree_mask=_as_words(self.sees).cuda(),
                    workspace=lynx.make_tree_workspace(self.geo, self.B, self.n, "cuda"))

    def exact(self, anchor=False, scale=None):
        """(out, lse, A, E) in 64 bits; E: bound of a score's error."""
        scale = 128 ** -0.5 if scale is None else scale
        B, n, Hkv, G, bt = self.B, self.n, self.Hkv, self.G, self.bt
        out = torch.zeros(B, n, Hkv * G, 128, dtype=torch.float64, device="cuda")
        lse, A, E = (torch.zeros(B, n, Hkv * G, dtype=torch.float64, device="cuda") for _ in range(3))
        for b, L in enumerate(self.lens):
            t = torch.arange(L)
            blk, off = self.table[b, t // bt].long(), t % bt
            vals, mags = [], []
            for p, x in zip(self.planes, (self.kn, self.vn)):
                a, r, m = (y[blk, :, off].cuda() for y in p)                         # [L][Hkv][..]
                level = 16 * _nibbles(a) + (8 if anchor else _nibbles(r))
                m = m.double()
                node = torch.where(self.sees[b].any(0)[:, None, None], x[b].double(), 0.0).cuda()
                vals.append(torch.cat((m[..., 1:] + m[..., :1] * level, node)))
                mags.append(torch.cat(((m[..., 1] + 128 * m[..., 0]).abs() + 128 * m[..., 0], node.abs().amax(-1))))
            allowed = torch.cat((torch.ones(n, L, dtype=torch.bool), self.sees[b]), 1).cuda()
            for h in range(Hkv):
                q = self.q[b, :, h * G:(h + 1) * G].double().cuda()
                s = torch.einsum("jgd,td->jgt", q, vals[0][:, h]) * scale
                s = s.masked_fill(~allowed[:, None], -math.inf)
                top = s.amax(-1, keepdim=True).clamp_min(-1e300)
                w = (s - top).exp()
                den = w.sum(-1, keepdim=True)
                w = torch.where(den > 0, w / den, 0.0)
                sl = slice(h * G, (h + 1) * G)
                out[b, :, sl] = w @ vals[1][:, h]
                lse[b, :, sl] = (den.log() + top)[..., 0]
                A[b, :, sl] = w @ mags[1][:, h]
                S = abs(scale) * q.abs().sum(-1) * mags[0][:, h].max()
                E[b, :, sl] = 2.0 ** -16 * S
        return out, lse, A, E


def _check(pr, anchor=False, scale=0.0, out_f32=False, dev=None):
    d = dev or pr.device()
    B, n, Hq = pr.q.shape[:3]
    lse = torch.full((B, n, Hq), 777.0, device="cuda")
    given = torch.full((B, n, Hq, 128), 777.0, device="cuda") if out_f32 else None
    got = lynx.tree_attention(**d, anchor_only=anchor, softmax_scale=scale, lse=lse, out=given)
    lynx.check(d["workspace"])
    out, want_lse, A, E = pr.exact(anchor, None if scale == 0.0 else scale)
    tol = (2.0 ** -9 + 2 * E) * A
    tol = tol[..., None] + (0.0 if out_f32 else 2.0 ** -8) * out.abs() + 1e-30
    err = (got.double() - out).abs()
    assert torch.isfinite(got).all()
    assert (err <= tol).all(), (err / tol).max().item()
    # and in the mean far below: a fifth of the bound's FP16 part
    if not out_f32 and out.numel() > 4096:
        assert err.norm().item() <= 4e-3 * out.norm().item()
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (got[empty] == 0).all()
    d_lse = (lse.double() - want_lse)[~empty].abs()
    assert (d_lse <= E[~empty] + 2.0 ** -18 * (1 + want_lse[~empty].abs())).all(), d_lse.max().item()
    return got


@pytest.mark.parametrize("lens", [(5,), (128,), (129,), (0, 1, 300)])
@pytest.mark.parametrize("n,G", [(1, 1), (1, 4), (7, 4), (16, 8)])
def test_small(lens, n, G):
    _check(Problem(lens, n, 2, G, seed=n + G))


@pytest.mark.parametrize("kind", ["tree", "chain", "random", "self", "none"])
@pytest.mark.parametrize("lens", [(0, 0), (0, 40), (700, 3)])
def test_masks(kind, lens):
    _check(Problem(lens, 33, 1, 4, kind=kind, seed=4))


@pytest.mark.parametrize("n,G,Hkv", [(2, 1, 1), (3, 2, 3), (13, 4, 8), (24, 4, 2), (32, 4, 2), (33, 4, 1), (64, 1, 2), (64, 8, 1), (64, 16, 1), (5, 7, 2)])
@pytest.mark.parametrize("lens", [(3000,), (100, 2111, 0, 640)])
@pytest.mark.parametrize("anchor", [False, True])
def test_columns_and_row_blocks(n, G, Hkv, lens, anchor):
    _check(Problem(lens, n, Hkv, G, seed=n), anchor=anchor)


@pytest.mark.parametrize("bt", [16, 32, 48, 128, 1024])
def test_block_sizes(bt):
    _check(Problem((777, 16, 2050), 9, 2, 4, bt=bt, seed=bt))


@pytest.mark.parametrize("lens,n,G,Hkv", [((40000,), 8, 4, 8), ((20000, 20000), 32, 4, 4), ((9000, 130, 4000, 17, 0, 25000), 12, 8, 2),
                                          (tuple([300] * 70), 6, 4, 1), (tuple(range(0, 4000, 61)), 20, 2, 2)])
def test_many_ctas(lens, n, G, Hkv):
    _check(Problem(lens, n, Hkv, G, seed=11))


def test_table_wider_than_the_sequences():
    _check(Problem((200, 1), 5, 2, 4, extra_blocks=600, seed=2))


@pytest.mark.parametrize("case", ["k_offset", "sharp", "flat_v", "big_v", "small_v", "uneven_v", "scale", "negative_scale"])
def test_values(case):
    kw = dict(k_offset=dict(k_off=20.0), sharp=dict(q_spread=12.0), flat_v=dict(v_rows=lambda z: torch.zeros_like(z)), big_v=dict(v_spread=1e30),
              small_v=dict(v_spread=1e-20), uneven_v=dict(v_rows=lambda z: torch.exp(3 * z))).get(case, {})
    pr = Problem((1500, 260), 11, 2, 4, seed=21, **kw)
    _check(pr, scale=dict(scale=0.31, negative_scale=-0.05).get(case, 0.0))
    _check(pr, out_f32=True, scale=dict(scale=0.31, negative_scale=-0.05).get(case, 0.0))


def test_rising_scores():
    """Scores that rise along the sequence by far more than a weight's range, so that every row's reference is raised again and again."""
    pr = Problem((6000,), 8, 1, 4, seed=31)
    a, r, m = pr.planes[0]
    t = torch.arange(6000)
    blk, off = pr.table[0, t // 16].long(), t % 16
    m[blk, :, off] *= (1 + t.float() / 100)[:, None, None]
    _check(pr)
    pr.q = pr.q.abs()
    _check(pr)


def test_same_call_again_other_shapes_and_streams():
    """A workspace serves calls of other lengths and batches; results do not depend on what it held."""
    pr, small = Problem((3000, 800), 24, 2, 4, seed=41), Problem((250, 31), 24, 2, 4, seed=42, extra_blocks=200)
    d, e = pr.device(), small.device()
    first = _check(pr, dev=d)
    e["workspace"] = d["workspace"]
    if lynx.tree_workspace_bytes(small.geo, 2, 24) <= d["workspace"].numel():
        _check(small, dev=e)
    again = lynx.tree_attention(**d)
    assert torch.equal(first, again)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        other = lynx.tree_attention(**d)
    st.synchronize()
    assert torch.equal(first, other)
    # captured and replayed
    out = torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lynx.tree_attention(**d, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)


def test_a_chain_is_a_verification():
    """The causal window of merge_verify_attention: its last k tokens as nodes.  Both are within their bounds of the exact result."""
    n, L, Hkv, G = 6, 500, 2, 4
    pr = Problem((L,), n, Hkv, G, kind="chain", seed=51)
    a = _check(pr, out_f32=True)
    # the same prefix by the other kernel, and the nodes by BF16 attention, joined
    d = pr.device()
    ws = lynx.make_workspace(pr.geo, 1, n, "cuda")
    for p in (d["K"], d["V"]):
        p.meta.nan_to_num_(0.0, 0.0)
    out, _, _ = lynx.merge_verify_attention(pr.geo, d["q"], d["K"], d["V"], d["block_table"], d["seq_lens"], ws, causal=False)
    lse = lynx.workspace_lse(pr.geo, 1, n, ws).clone()
    tail_geo = lynx.Geometry(Hkv * G, Hkv, 16, 1, 1)
    pages = []
    for x in (pr.kn, pr.vn):
        y = torch.zeros(1, Hkv, 16, 128, dtype=torch.bfloat16)
        y[0, :, :n] = x[0].transpose(0, 1)
        pages.append(y.cuda())
    tws = torch.empty(int(lynx.load().lynx_bf16_workspace_bytes(lynx.ctypes.byref(tail_geo._c()), 1, n)), dtype=torch.uint8, device="cuda")
    tail = lynx.bf16_attention(tail_geo, d["q"], *pages, torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                               torch.tensor([n], dtype=torch.int32, device="cuda"), tws, causal=True)
    both = lynx.lse_merge(out, lse, tail, lynx.bf16_workspace_lse(tail_geo, 1, n, tws))
    _, _, A, E = pr.exact()
    assert ((a - both).abs().double() <= 2 * ((2.0 ** -9 + 2 * E) * A)[..., None] + 2e-3).all()


def test_the_extension_and_the_python_body_agree(monkeypatch):
    pr = Problem((300, 0, 41), 6, 2, 4, seed=81)
    d = pr.device()
    lse = [torch.empty(3, 6, 8, device="cuda") for _ in range(2)]
    fast = lynx.tree_attention(**d, lse=lse[0]), lynx.tree_attention(**d, anchor_only=True, out=torch.empty(d["q"].shape, device="cuda"))
    monkeypatch.setattr(lynx, "_fast_tree_attention", lynx._python_only)
    slow = lynx.tree_attention(**d, lse=lse[1]), lynx.tree_attention(**d, anchor_only=True, out=torch.empty(d["q"].shape, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(fast + (lse[0],), slow + (lse[1],)))


def test_bad_block_ids_are_reported():
    pr = Problem((100, 50), 4, 1, 4, seed=61)
    d = pr.device()
    d["block_table"][1, 2] = 10 ** 6
    for p in (d["K"], d["V"]):
        p.meta.nan_to_num_(0.0, 0.0)
    lynx.tree_attention(**d)
    with pytest.raises(lynx.LynxError, match="block id"):
        lynx.check(d["workspace"])
    lynx.check(d["workspace"])


def test_refusals():
    pr = Problem((100, 50), 4, 2, 4, seed=71)
    d = pr.device()
    def bad(**kw):
        with pytest.raises((lynx.LynxError, RuntimeError)):
            lynx.tree_attention(**{**d, **kw})
    bad(q=d["q"].float())
    bad(q=d["q"][..., :64])
    bad(q=d["q"][:, :3])                                          # other nodes than the mask's
    bad(q=d["q"].transpose(0, 1))
    bad(block_table=d["block_table"].long())
    bad(seq_lens=d["seq_lens"][:1])
    bad(tree_mask=d["tree_mask"].int())
    bad(k_nodes=d["k_nodes"].float())
    bad(k_nodes=d["k_nodes"][:, :, :1])
    bad(v_nodes=d["v_nodes"].transpose(0, 1).contiguous().transpose(0, 1))     # nodes not evenly apart
    bad(workspace=d["workspace"][:-256])
    bad(K=lynx.Planes(d["K"].anchor, None, d["K"].meta))
    bad(out=torch.empty(d["q"].shape, dtype=torch.float16, device="cuda"))
    bad(lse=torch.empty(2, 4, 8, 1, device="cuda"))
    bad(geo=lynx.Geometry(8, 2, 24, pr.geo.num_blocks, pr.geo.max_blocks_per_seq))
    assert lynx.tree_workspace_bytes(pr.geo, 2, 65) == 0 and lynx.tree_workspace_bytes(lynx.Geometry(34, 2, 16, 4, 4), 1, 1) == 0
    with pytest.raises(lynx.LynxError):
        lynx.make_tree_workspace(pr.geo, 2, 65, "cuda")
    got = lynx.tree_attention(**{**d, "q": d["q"][:0], "block_table": d["block_table"][:0], "seq_lens": d["seq_lens"][:0],
                                 "tree_mask": d["tree_mask"][:0], "k_nodes": d["k_nodes"][:0], "v_nodes": d["v_nodes"][:0]})
    assert got.shape[0] == 0
