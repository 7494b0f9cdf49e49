"""The hand-offs of the tree attention kernel's roles, played through on the host: barriers that count arrivals and know a parity, roles
that run in any order, pieces of any length.  A wait that looks for a phase which its barrier has left behind by two would never
end; neither would a circle of roles.  Also what is handed over: nobody writes a place that somebody still reads."""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01831_b200", "csrc")


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1

    def done(self, parity):          # what the hardware answers
        return (self.phase & 1) != (parity & 1)


class Place:
    """Written by a role for a tile, read by others of the same tile."""
    def __init__(self, name):
        self.name, self.tile, self.readers = name, None, 0

    def write(self, tile):
        assert self.readers == 0, f"{self.name} of {self.tile} overwritten while it is read"
        self.tile = tile

    def read(self, tile):
        assert self.tile == tile, f"{self.name}: {self.tile} instead of {tile}"


N = 3       # places for scores and tiles


def _run(pieces, ring_k, ring_v, rng, softmax=4):
    """pieces: (tiles, whether the last is the nodes').  Warps of a role that only arrive together are one here."""
    B = {}
    for name, n, count in (("kfull", ring_k, 1), ("kempty", ring_k, 2), ("vfull", ring_v, 1), ("vempty", ring_v, 2), ("kready", N, 1), ("sfull", N, 1),
                           ("mready", 8, 1), ("vready", N, 1), ("pready", N, softmax), ("pvdone", N, 1), ("ifull", 2, 1),
                           ("iempty", 2, 2 * softmax + 5), ("qready", 2, 1), ("kdone", 2, 1)):
        B[name] = [Barrier(count) for _ in range(n)]
    rawk, rawv = [Place(f"raw K {i}") for i in range(ring_k)], [Place(f"raw V {i}") for i in range(ring_v)]
    ktile, vtile, vm, km, mids, S = ([Place(f"{x} {i}") for i in range(N)] for x in ("K", "V", "vm", "km", "mid", "S"))
    factor, exp = ([Place(f"{x} {i}") for i in range(8)] for x in ("a", "e"))
    item, O, Q = [Place("item 0"), Place("item 1")], [Place("O 0"), Place("O 1")], Place("Q")
    pair = [[0, 0] for _ in range(softmax)]         # arrivals of a row's two warps at the barriers at the end of a piece
    issued = []        # products, in order, completed in order

    def wait(bar, i, parity):
        while not B[bar][i].done(parity):
            yield
        yield

    def get(ic):
        yield from wait("ifull", ic & 1, ic >> 1)
        item[ic & 1].read(ic)
        return pieces[ic] if ic < len(pieces) else (0, False)

    def raw_tiles(n, tree):
        return n - 1 if tree else n

    def copies(k_side):
        full, empty, ring, place = ("kfull", "kempty", ring_k, rawk) if k_side else ("vfull", "vempty", ring_v, rawv)
        slot, phase, t, gs = 0, 1, 0, 0
        for ic in range(len(pieces) + 1):
            if k_side:
                yield from wait("iempty", ic & 1, (ic >> 1) - 1)
                item[ic & 1].write(ic)
                B["ifull"][ic & 1].arrive()
                n, tree = pieces[ic] if ic < len(pieces) else (0, False)
            else:
                n, tree = yield from get(ic)
            if n == 0:
                return
            for _ in range(raw_tiles(n, tree)):
                yield from wait(empty, slot, phase)
                place[slot].write(gs)
                B[full][slot].arrive()
                gs += 1
                slot, phase = (0, phase ^ 1) if slot + 1 == ring else (slot + 1, phase)
            gs += tree
            if not k_side:
                B["iempty"][ic & 1].arrive()

    def k_tiles():
        gs = slot = 0
        for ic in range(len(pieces) + 1):
            n, tree = yield from get(ic)
            if n == 0:
                return
            if gs > 0:
                yield from wait("sfull", (gs - 1) % N, (gs - 1) // N)
            Q.write(ic)
            B["qready"][ic & 1].arrive()
            for u in range(n):
                g = gs % N
                yield from wait("mready", gs & 7, gs >> 3)
                ktile[g].write(gs)
                if u < raw_tiles(n, tree):
                    rawk[slot].read(gs)
                    km[g].read(gs)
                    km[g].readers += 1
                    yield
                    km[g].readers -= 1
                    B["kempty"][slot].arrive()
                    slot = (slot + 1) % ring_k
                else:
                    factor[gs & 7].write(gs)
                    mids[g].write(gs)
                B["kready"][g].arrive()
                gs += 1
            B["kdone"][ic & 1].arrive()
            B["iempty"][ic & 1].arrive()

    def v_tiles():
        gs = slot = 0
        for ic in range(len(pieces) + 1):
            n, tree = yield from get(ic)
            if n == 0:
                return
            for u in range(n):
                g = gs % N
                yield from wait("mready", gs & 7, gs >> 3)
                yield from wait("pvdone", g, gs // N - 1)
                vtile[g].write(gs)
                if u < raw_tiles(n, tree):
                    rawv[slot].read(gs)
                    vm[g].read(gs)
                    vm[g].readers += 1
                    yield
                    vm[g].readers -= 1
                    B["vempty"][slot].arrive()
                    slot = (slot + 1) % ring_v
                else:
                    exp[gs & 7].write(gs)
                B["vready"][g].arrive()
                gs += 1
            B["iempty"][ic & 1].arrive()

    def scales():
        gs = ks = kp = vs = vp = 0
        for ic in range(len(pieces) + 1):
            n, tree = yield from get(ic)
            if n == 0:
                return
            yield from wait("qready", ic & 1, ic >> 1)
            for u in range(n):
                g = gs % N
                prefix = u < raw_tiles(n, tree)
                if prefix:
                    yield from wait("kfull", ks, kp)
                    yield from wait("vfull", vs, vp)
                    rawk[ks].read(gs)
                    rawv[vs].read(gs)
                    B["kempty"][ks].arrive()
                    B["vempty"][vs].arrive()
                    ks, kp = (0, kp ^ 1) if ks + 1 == ring_k else (ks + 1, kp)
                    vs, vp = (0, vp ^ 1) if vs + 1 == ring_v else (vs + 1, vp)
                yield from wait("sfull", g, gs // N - 1)
                yield from wait("vready", g, gs // N - 1)
                if prefix:
                    for x in (km[g], vm[g], mids[g], exp[gs & 7], factor[gs & 7]):
                        x.write(gs)
                B["mready"][gs & 7].arrive()
                gs += 1
            B["iempty"][ic & 1].arrive()

    def products():
        ahead = gs = 0

        def qk(ic):
            nonlocal ahead
            yield from wait("kready", ahead % N, ahead // N)
            Q.readers += 1
            ktile[ahead % N].readers += 1
            mids[ahead % N].readers += 1
            issued.append(("qk", ahead, ic, False))
            ahead += 1

        for ic in range(len(pieces) + 1):
            n, _ = yield from get(ic)
            if n == 0:
                return
            end = gs + n
            while ahead < min(end, gs + N):
                yield from qk(ic)
            for u in range(n):
                yield from wait("vready", gs % N, gs // N)
                yield from wait("pready", gs % N, gs // N)
                vtile[gs % N].readers += 1
                issued.append(("pv", gs, ic, u < 2))
                gs += 1
                if ahead < end:
                    yield from qk(ic)
            B["iempty"][ic & 1].arrive()

    def tensor_core():
        while True:
            if not issued:
                yield
                continue
            kind, gs, ic, first = issued[0]      # (in order, one behind the other)
            g = gs % N
            if kind == "qk":
                S[g].write(gs)
            elif first:
                O[gs & 1].write(ic)
            yield
            issued.pop(0)
            if kind == "qk":
                Q.read(ic)
                ktile[g].read(gs)
                mids[g].read(gs)
                mids[g].readers -= 1
                Q.readers -= 1
                ktile[g].readers -= 1
                B["sfull"][g].arrive()
            else:
                S[g].read(gs)
                vtile[g].read(gs)
                O[gs & 1].read(ic)
                vtile[g].readers -= 1
                B["pvdone"][g].arrive()

    def softmax_warp(group, w):
        gs = turn = 0
        for ic in range(len(pieces) + 1):
            n, tree = yield from get(ic)
            if n == 0:
                return
            first = True
            for u in range(n):
                if gs & 1 != group:
                    gs += 1
                    continue
                g = gs % N
                yield from wait("mready", gs & 7, gs >> 3)
                if tree and u == n - 1:
                    yield from wait("kdone", ic & 1, ic >> 1)
                    yield from wait("vready", g, gs // N)
                yield from wait("sfull", g, gs // N)
                places = (S[g], factor[gs & 7], exp[gs & 7])
                for p in places:
                    p.read(gs)
                    p.readers += 1
                yield
                if not first and rng.random() < 0.2:      # the reference is raised
                    yield from wait("pvdone", (gs - 2) % N, (gs - 2) // N)
                for p in places:
                    p.readers -= 1
                B["pready"][g].arrive()
                first = False
                gs += 1
            yield from wait("pvdone", (gs - 1) % N, (gs - 1) // N)
            if n > 1:
                yield from wait("pvdone", (gs - 2) % N, (gs - 2) // N)
            used = O[:] if n > 1 else [O[(gs - 1) & 1]]
            for o in used:
                o.read(ic)
                o.readers += 1
            yield
            for o in used:
                o.readers -= 1
            turn += 1
            pair[w][group] = turn
            while pair[w][group ^ 1] < turn:              # (the two warps of a row)
                yield
            B["iempty"][ic & 1].arrive()

    roles = [copies(True), copies(False), k_tiles(), v_tiles(), scales(), products()] + [softmax_warp(g, w) for g in range(2) for w in range(softmax)]
    core = tensor_core()
    speed = [rng.choice([1, 1, 1, 3, 30, 200]) for _ in roles]
    core_speed, idle = rng.choice([1, 3, 30]), 0
    while roles:
        before = [(b.phase, b.left) for bs in B.values() for b in bs], len(issued)
        for i in rng.sample(range(len(roles)), len(roles)):
            if rng.random() * speed[i] < 1:
                try:
                    next(roles[i])
                except StopIteration:
                    roles[i] = None
        if rng.random() * core_speed < 1:
            next(core)
        keep = [i for i, r in enumerate(roles) if r is not None]
        roles, speed = [roles[i] for i in keep], [speed[i] for i in keep]
        idle = idle + 1 if before == ([(b.phase, b.left) for bs in B.values() for b in bs], len(issued)) else 0
        assert idle < 20000, "nobody moves"
    assert not issued


@pytest.mark.parametrize("rings", [(7, 6), (2, 5), (1, 1)])
def test_every_role_ends(rings):
    rng = random.Random(9)
    for _ in range(20):
        pieces = [(rng.choice([1, 1, 2, 3, 4, 7, 12]), rng.random() < 0.5) for _ in range(rng.randint(1, 6))]
        _run(pieces, *rings, rng, softmax=rng.choice([1, 4]))


def test_the_kernel_waits_for_what_is_played():
    """The waits of the roles in the source, by barrier."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "tree_attention.cu")).read())
    code = code[code.index("tree_attention_kernel("):code.index("tree_combine_kernel(")]
    cuts = ["if (warp < 8) {", "if (warp < 12) {", "if (warp < 16) {", "if (warp < 18) {", "if (warp == 19) {", "if (warp == 18) {"]
    at = [code.index(x) for x in cuts] + [len(code)]
    waits = [sorted(set(re.findall(r"\bwait\((\w+)", code[a:b]))) for a, b in zip(at, at[1:])]
    assert waits == [["ifull", "kdone", "mready", "pvdone", "sfull", "vready"], ["ifull", "mready", "sfull"],
                     ["ifull", "mready", "pvdone"], ["empty", "iempty", "ifull"],
                     ["ifull", "kfull", "qready", "sfull", "vfull", "vready"], ["ifull", "kready", "pready", "vready"]]
    land, done, free = (code.index(x) for x in ("land_after_abort(", "named_bar(2, kDoneThreads)", "tcgen05.dealloc"))
    assert done < land < free and len(re.findall(r"bar_arrive\(2, kDoneThreads\)", code)) == 2
