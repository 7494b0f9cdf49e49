"""Block tables, slots and positions from lengths, against loops over requests and tokens: whole numbers, all equal."""
import random

import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu


class Pool:
    """The plan in loops: a queue of free blocks in a ring."""

    def __init__(self, geo, ring, head, count, table):
        self.geo, self.ring, self.head, self.count, self.table = geo, list(ring), head, count, [list(r) for r in table]

    def plan(self, old, new, max_tokens):
        bt, P, cap = self.geo.block_tokens, self.geo.num_blocks, self.geo.max_blocks_per_seq * self.geo.block_tokens
        old, new = [min(max(n, 0), cap) for n in old], [min(max(n, 0), cap) for n in new]
        wanted = taken = given = 0
        lens, offsets, slots, positions = [], [0], [], []
        freed = []
        for b, (a, n) in enumerate(zip(old, new)):
            have, want = -(-a // bt), -(-n // bt)
            need = max(0, want - have)
            wanted += need
            ok = need == 0 or wanted <= self.count
            if ok:
                for k in range(need):
                    self.table[b][have + k] = self.ring[(self.head + taken + k) % P]
                taken += need
                freed += self.table[b][want:have]
            lens.append(n if ok else a)
            for t in range(a, n):
                blk = self.table[b][t // bt]
                slots.append(blk * bt + t % bt if ok and 0 <= blk < P else -1)
                positions.append(t)
            offsets.append(len(positions))
        for i, blk in enumerate(freed):
            self.ring[(self.head + self.count + i) % P] = blk
        self.head, self.count = (self.head + taken) % P, self.count - taken + len(freed)
        pad = max(0, max_tokens - len(slots))
        return lens, offsets, (slots + [-1] * pad)[:max_tokens], (positions + [0] * pad)[:max_tokens]


def _step(geo, pool, table, model, old, new, rows):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    got = lynx.plan_blocks(geo, pool, table, i32(old), i32(new), rows)
    want = model.plan(old, new, rows)
    for name, g, w in zip(lynx.BlockPlan._fields, got, want):
        assert g.tolist() == w, name
    assert pool.ring.tolist() == model.ring and pool.state.tolist() == [model.head, model.count, 0, 0]
    assert table.tolist() == model.table
    return got.lens.tolist()


def _make(B, bt, nb, mb, head=0):
    geo = lynx.Geometry(8, 8, bt, nb, mb)
    ring = torch.arange(nb, dtype=torch.int32).roll(head)
    pool = lynx.BlockPool(ring.cuda(), torch.tensor([head, nb, 0, 0], dtype=torch.int32).cuda())
    table = torch.full((B, mb), -7, dtype=torch.int32).cuda()
    return geo, pool, table, Pool(geo, ring.tolist(), head, nb, table.tolist())


@pytest.mark.parametrize("B", [1, 3, 64, 1000, 1024, 1025, 2600])
@pytest.mark.parametrize("bt", [1, 5, 16, 64])
def test_a_life_of_requests(B, bt):
    """Admission, decode steps, windows taken back, requests that end and rows that start anew; the ring goes round."""
    r = random.Random(B * 100 + bt)
    mb = 200 // bt + 2
    nb = B * mb // 2 + 3
    geo, pool, table, model = _make(B, bt, nb, mb, head=r.randrange(nb))
    lens = [0] * B
    for step in range(6):
        new = [r.choice([n, n + 1, n + 4, max(0, n - 3), 0, r.randint(0, mb * bt)]) if step else r.randint(0, 100) for n in lens]
        total = sum(max(0, b - a) for a, b in zip(lens, new))
        lens = _step(geo, pool, table, model, lens, new, r.choice([total, total + 7, total // 2, 0, total + 2000]))
    assert B == 1 or model.count < nb          # (some hold blocks)
    lens = _step(geo, pool, table, model, lens, [0] * B, 5)
    assert lens == [0] * B and model.count == nb and sorted(model.ring) == list(range(nb))


@pytest.mark.parametrize("free", [0, 1, 9, 10, 11])
def test_too_few_free_blocks(free):
    """Requests from the first that does not fit on get nothing, those that need none go on."""
    bt, B = 16, 6
    geo, pool, table, model = _make(B, bt, 40, 8)
    lens = _step(geo, pool, table, model, [0] * B, [16, 20, 1, 0, 30, 16], 100)      # 1 + 2 + 1 + 0 + 2 + 1 blocks
    lens = _step(geo, pool, table, model, lens, [16, 20, 1, 0, 30, 128], 112)        # all but 40 - 7 - 7 = 26
    model.count = free
    pool.state[1] = free
    got = _step(geo, pool, table, model, lens, [17, 64, 16, 90, 32, 100], 200)       # 1, 2, 0, 6, 0, -1 blocks; 9 in all
    assert got == ([17, 64, 16, 90, 32, 100] if free >= 9 else [17, 20, 16, 0, 32, 100] if free == 1 else [16, 20, 16, 0, 32, 100])


def test_one_long_prompt_among_many():
    B, bt = 300, 16
    geo, pool, table, model = _make(B, bt, 6000, 4097)
    lens = _step(geo, pool, table, model, [0] * B, [5] * 7 + [65535] + [3] * (B - 8), 70001)
    _step(geo, pool, table, model, lens, [6] * 7 + [0] + [17] * (B - 8), 0)


def test_lengths_and_ids_out_of_range():
    bt, mb = 16, 4
    geo, pool, table, model = _make(4, bt, 30, mb)
    lens = _step(geo, pool, table, model, [-5, 0, 0, 0], [3, 1000, -1, 64], 140)
    assert lens == [3, 64, 0, 64]
    table[0, 0], model.table[0][0] = 99, 99       # an id that is none of the pool's: its tokens have no slot
    _step(geo, pool, table, model, lens, [9, 64, 5, 64], 16)


def test_no_requests():
    geo, pool, table, model = _make(0, 16, 5, 3)
    _step(geo, pool, table, model, [], [], 0)
    _step(geo, pool, table, model, [], [], 9)


def test_other_outputs_alignments_and_streams(monkeypatch):
    """Outputs left out, outputs that begin at an odd place, the Python body, a side stream."""
    B, bt = 5, 16
    L, i32 = lynx.load(), lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    for variant in range(3):
        geo, pool, table, model = _make(B, bt, 60, 9)
        old, new = [0] * B, [40, 3, 0, 100, 17]
        want = model.plan(old, new, 150)
        lens, offsets = i32([0] * B), i32([0] * (B + 1))
        slots, positions = torch.full((152,), 5, dtype=torch.int64).cuda(), torch.full((152,), 5, dtype=torch.int32).cuda()
        a = i32(old), i32(new)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        ptr = lambda t: t.data_ptr()
        assert L.lynx_plan_blocks(ctypes_shape(geo), ptr(a[0]), ptr(a[1]), B, ptr(table), ptr(pool.ring), ptr(pool.state), 150, ptr(lens),
                                  ptr(offsets) if variant != 1 else None, ptr(slots[1:]) if variant != 2 else None,
                                  ptr(positions[1:]) if variant != 1 else None, st.cuda_stream) == 0
        st.synchronize()
        assert lens.tolist() == want[0] and table.tolist() == model.table and pool.ring.tolist() == model.ring
        assert offsets.tolist() == (want[1] if variant != 1 else [0] * (B + 1))
        assert slots.tolist() == ([5] + want[2] + [5] if variant != 2 else [5] * 152)
        assert positions.tolist() == ([5] + want[3] + [5] if variant != 1 else [5] * 152)
    monkeypatch.setattr(lynx, "_fast_plan_blocks", lynx._python_only)
    geo, pool, table, model = _make(B, bt, 60, 9)
    _step(geo, pool, table, model, [0] * B, [40, 3, 0, 100, 17], 150)


def ctypes_shape(geo):
    import ctypes
    return ctypes.byref(geo._c())


def test_captured_and_replayed():
    """A decode step in a graph: each replay takes up where the last one left off."""
    B, bt = 8, 16
    geo, pool, table, model = _make(B, bt, 100, 12)
    old, new = torch.zeros(B, dtype=torch.int32).cuda(), torch.zeros(B, dtype=torch.int32).cuda()
    lynx.plan_blocks(geo, pool, table, old, new, 16)
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        new.copy_(old + 3)
        plan = lynx.plan_blocks(geo, pool, table, old, new, 32)
        old.copy_(plan.lens)
    lens = [0] * B
    for _ in range(12):
        graph.replay()
        want = model.plan(lens, [n + 3 for n in lens], 32)
        assert [x.tolist() for x in plan] == list(want)
        lens = want[0]
        assert old.tolist() == lens and table.tolist() == model.table and pool.ring.tolist() == model.ring
