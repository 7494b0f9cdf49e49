"""The calls around a decode step together, for models that norm their heads: plans, norms with positions, keys normed into the cache, attention over what
was written, ranges read back; eager, and as one captured step that is replayed with other lengths."""
import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu
HQ, HKV, BT, EPS = 8, 2, 16, 1e-6


class Model:
    """A layer's keys and values by request and position, made up beforehand, and the cache that they go into."""

    def __init__(self, B, capacity, blocks, seed):
        g = torch.Generator().manual_seed(seed)
        self.B, self.capacity = B, capacity
        self.q, self.k, self.v = (torch.randn(B, capacity, h, 128, generator=g).to(torch.bfloat16).cuda() for h in (HQ, HKV, HKV))
        self.norm = lynx.HeadNorm(*((1 + 0.2 * torch.randn(128, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)), EPS)
        self.angles = lynx.rotary_table(capacity, 64, device="cuda")
        self.geo = lynx.Geometry(HQ, HKV, BT, blocks, -(-capacity // BT))
        self.K, self.V = (lynx.Planes(torch.zeros(blocks, HKV, BT, 64, dtype=torch.uint8, device="cuda"),
                                      torch.zeros(blocks, HKV, BT, 64, dtype=torch.uint8, device="cuda"), torch.zeros(blocks, HKV, BT, 2, device="cuda"))
                          for _ in range(2))
        self.pool = lynx.make_block_pool(blocks, "cuda")
        self.table = torch.full((B, self.geo.max_blocks_per_seq), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.ws = lynx.make_tree_workspace(self.geo, B, 1, "cuda")
        self.node = torch.zeros(B, 1, HKV, 128, dtype=torch.bfloat16, device="cuda")
        self.none = torch.zeros(B, 1, dtype=torch.int64, device="cuda")     # (a tree without nodes: the prefix alone)

    def step(self, new_lens, max_tokens):
        """-> the plan, what the cache held before, the new tokens as read back, and the last positions' queries and attention."""
        before = self.lens.clone()
        plan = lynx.plan_blocks(self.geo, self.pool, self.table, before, new_lens, max_tokens)
        # the new tokens' rows; padding behind the last, which has no slot, is some row
        row = torch.arange(max_tokens, device="cuda", dtype=torch.int32)
        b = (torch.searchsorted(plan.offsets, row, right=True) - 1).clamp(0, self.B - 1)
        at = plan.positions.long().clamp(max=self.capacity - 1)
        k, v = self.k[b, at], self.v[b, at]
        spec = lynx.Rotary(plan.positions, self.angles)
        lynx.cache_append(self.geo, k, v, plan.slots, self.K, self.V, rotary=spec, norm=self.norm)
        last = (plan.lens - 1).clamp(min=0)
        q = lynx.norm_rotary(self.q[torch.arange(self.B, device="cuda"), last.long()], None, self.norm, lynx.Rotary(last, self.angles))[0]
        out = lynx.tree_attention(self.geo, q[:, None], self.K, self.V, self.table, plan.lens, self.node, self.node, self.none, self.ws)
        back = lynx.cache_read(self.geo, self.K, self.V, self.table, before, plan.offsets, max_tokens)
        self.lens.copy_(plan.lens)
        return plan, before, back, q, out[:, 0]

    def turned(self, x, weight, at):
        """x [n][heads][128] normed and turned to positions at [n], 64 bits."""
        x = x.double()
        if weight is not None:
            x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
        c, s = (t[:, None] for t in self.angles[at].double().split(64, 1))
        return torch.cat((x[..., :64] * c - x[..., 64:] * s, x[..., 64:] * c + x[..., :64] * s), -1)

    def check(self, asked, plan, before, back, q, out):
        before, asked, lens = before.tolist(), asked.tolist(), plan.lens.tolist()
        lynx.check(self.ws)
        held = [-(-n // BT) for n in lens]
        used = [i for b, n in enumerate(held) for i in self.table[b, :n].tolist()]
        assert len(set(used)) == len(used) and int(self.pool.state[1]) == self.geo.num_blocks - len(used)
        row = 0
        for b, (old, want, now) in enumerate(zip(before, asked, lens)):
            assert now in (old, want) and plan.offsets[b] == row
            grown = max(want - old, 0)
            if now == want and grown:           # what was written: half a step of 8 bits, the rounding of what is read to BF16, FP32's own
                t = torch.arange(old, now, device="cuda")
                for got, exact in ((back[0], self.turned(self.k[b, t], self.norm.k_weight, t)), (back[1], self.v[b, t].double())):
                    span, most = exact.amax(-1, keepdim=True) - exact.amin(-1, keepdim=True), exact.abs().amax(-1, keepdim=True)
                    assert ((got[row:row + grown].double() - exact).abs() <= span * (1 + 2.0 ** -6) / 510 + (2.0 ** -8 + 2.0 ** -20) * most).all()
            row += grown
        assert int(plan.offsets[self.B]) == row
        # attention over what the planes hold: bounds as for decoding with trees
        keys, vals = (p.meta[..., 1:].double() + p.meta[..., :1].double() * lynx.recombine(p)[0].double() for p in (self.K, self.V))
        for b, n in enumerate(lens):
            if n == 0:
                assert (out[b] == 0).all()
                continue
            blk, t = self.table[b].long(), torch.arange(n, device="cuda")
            kx, vx = (x[blk[t // BT], :, t % BT].repeat_interleave(HQ // HKV, 1) for x in (keys, vals))
            exact = self.turned(self.q[b, n - 1][None], self.norm.q_weight, t[-1:])[0]
            assert ((q[b].double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 2.0 ** -20 * exact.abs().amax(-1, keepdim=True)).all()
            p = (torch.einsum("hd,thd->ht", q[b].double(), kx) / 128 ** 0.5).softmax(-1)
            want = torch.einsum("ht,thd->hd", p, vx)
            size_k, size_v = (2 * x.abs().max() for x in (kx, vx))
            E = 2.0 ** -16 * q[b].double().abs().sum(-1).max() * size_k / 128 ** 0.5      # of a score
            assert ((out[b].double() - want).abs() <= (2.0 ** -9 + 2 * E) * size_v + 2.0 ** -8 * want.abs()).all()


LENGTHS = [(5, 0, 64, 33, 16), (6, 1, 65, 34, 17), (7, 2, 66, 35, 18), (0, 90, 66, 36, 19), (40, 91, 3, 37, 19), (41, 92, 4, 0, 60), (90, 92, 70, 80, 96)]


def test_requests_of_all_kinds_in_turn():
    m = Model(5, 96, 22, 1)     # (22 blocks of 16: the last lengths do not all fit)
    for lens in LENGTHS:
        asked = torch.tensor(lens, dtype=torch.int32).cuda()
        m.check(asked, *m.step(asked, 400))
    assert m.lens.tolist() != list(LENGTHS[-1])


def test_one_captured_step():
    m, eager = Model(5, 96, 22, 1), Model(5, 96, 22, 1)
    asked = torch.tensor(LENGTHS[0], dtype=torch.int32).cuda()
    warm = Model(5, 96, 22, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step(asked, 400)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = m.step(asked, 400)
    for lens in LENGTHS:
        asked.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        m.check(asked, *result)
        plan, _, back, _, out = eager.step(asked, 400)
        rows = int(plan.offsets[-1])
        assert torch.equal(out, result[4]) and torch.equal(plan.slots, result[0].slots)
        assert all(torch.equal(x[:rows], y[:rows]) for x, y in zip(back, result[2]))
