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


N = 3       # places for scores, and for the scales of a tile


def _halves(n, tree, short):
    """Half tiles of a piece of n tiles: (tile, whether it is its tile's first, its last).  short: the prefix ends in a first half."""
    out = []
    for t in range(n - 1 if tree else n):
        one = short and t == (n - 2 if tree else n - 1)
        out += [(t, True, one)] + ([] if one else [(t, False, True)])
    return out + ([(n - 1, True, True)] if tree else [])


def _run(pieces, ring_k, ring_v, rng, softmax=4):
    """pieces: (tiles, whether the last is the nodes', whether the prefix ends in the first half of a tile).  Warps of a role that
    only arrive together are one here."""
    B = {}
    for name, n, count in (("kfull", ring_k, 1), ("kempty", ring_k, 2), ("vfull", ring_v, 1), ("vempty", ring_v, 2), ("kready", 2, 2), ("sfull", N, 1),
                           ("mready", 8, 2), ("vready", N, 2), ("pready", N, softmax), ("pvdone", N, 1), ("kfree", N, 1), ("vfree", 2, 1),
                           ("ifull", 2, 1), ("iempty", 2, 2 * softmax + 7), ("qready", 2, 4), ("kdone", 2, 1), ("kscales", N, 1), ("vscales", N, 1)):
        B[name] = [Barrier(count) for _ in range(n)]
    rawk, rawv = [Place(f"raw K {i}") for i in range(ring_k)], [Place(f"raw V {i}") for i in range(ring_v)]
    S = [Place(f"S {i}") for i in range(N)]
    vm, km, mids = ([Place(f"{x} {i}") for i in range(N)] for x in ("vm", "km", "mid"))
    ktile, vtile = ([[Place(f"{x} {i} {j}") for j in range(2)] for i in range(2)] for x in ("K", "V"))
    factor, exp = ([Place(f"{x} {i}") for i in range(n)] for x, n in (("a", 2 * N), ("e", 8)))
    item, O, Q = [Place("item 0"), Place("item 1")], [Place("O 0"), Place("O 1")], [Place(f"Q {i}") for i in range(4)]
    maxima, met = [[Place(f"maxima {i} {j}") for j in range(4)] for i in range(2)], [0] * 4       # of the queries; barriers of the roles that have them
    pair = [[0, 0] for _ in range(softmax)]         # arrivals of a row's two warps at the barriers at the end of a piece
    issued = []        # products, in order, completed in order

    def wait(bar, i, parity):
        while not B[bar][i].done(parity):
            yield
        yield

    def get(ic):
        yield from wait("ifull", ic & 1, ic >> 1)
        item[ic & 1].read(ic)
        return pieces[ic] if ic < len(pieces) else (0, False, False)

    def meet(i):
        met[i] += 1
        while min(met) < met[i]:
            yield

    def queries(i, ic, gt):
        maxima[ic & 1][i].write(ic)
        yield from meet(i)
        for m in maxima[ic & 1]:
            m.read(ic)
            m.readers += 1
        yield
        for m in maxima[ic & 1]:
            m.readers -= 1
        if gt > 0:
            yield from wait("kfree", (gt - 1) % N, (gt - 1) // N)
        Q[i].write(ic)
        yield from meet(i)
        if i == 0:
            for q in Q:                     # (the sums of all quarters)
                q.read(ic)
            Q[0].write(ic)
        B["qready"][ic & 1].arrive()

    def raw_tiles(n, tree):
        return n - 1 if tree else n

    def copies():
        ks, vs, kp, vp, gt = 0, 0, 1, 1, 0
        for ic in range(len(pieces) + 1):
            yield from wait("iempty", ic & 1, (ic >> 1) - 1)
            item[ic & 1].write(ic)
            B["ifull"][ic & 1].arrive()
            n, tree, _ = pieces[ic] if ic < len(pieces) else (0, False, False)
            if n == 0:
                return
            for _ in range(raw_tiles(n, tree)):
                yield from wait("kempty", ks, kp)
                rawk[ks].write(gt)
                B["kfull"][ks].arrive()
                yield from wait("vempty", vs, vp)
                rawv[vs].write(gt)
                B["vfull"][vs].arrive()
                gt += 1
                ks, kp = (0, kp ^ 1) if ks + 1 == ring_k else (ks + 1, kp)
                vs, vp = (0, vp ^ 1) if vs + 1 == ring_v else (vs + 1, vp)
            gt += tree

    def k_tiles(side):
        gt = slot = phase = 0
        for ic in range(len(pieces) + 1):
            n, tree, short = yield from get(ic)
            if n == 0:
                return
            yield from queries(side, ic, gt)
            for u in range(n):
                g = gt & 1
                yield from wait("kscales", gt % N, gt // N)
                if gt > 1:
                    yield from wait("kfree", (gt - 2) % N, (gt - 2) // N)
                if u < raw_tiles(n, tree):
                    yield from wait("kfull", slot, phase)
                    ktile[g][side].write(gt)
                    rawk[slot].read(gt)
                    km[gt % N].read(gt)
                    km[gt % N].readers += 1
                    yield
                    km[gt % N].readers -= 1
                    B["kempty"][slot].arrive()
                    slot, phase = (0, phase ^ 1) if slot + 1 == ring_k else (slot + 1, phase)
                elif side == 0:
                    ktile[g][0].write(gt)
                    factor[gt % (2 * N)].write(gt)
                    mids[gt % N].write(gt)
                B["kready"][g].arrive()
                gt += 1
            if side == 0:
                B["kdone"][ic & 1].arrive()
            B["iempty"][ic & 1].arrive()

    def v_tiles(side):
        gt = slot = phase = 0
        for ic in range(len(pieces) + 1):
            n, tree, short = yield from get(ic)
            if n == 0:
                return
            yield from queries(2 + side, ic, gt)
            for u in range(n):
                g = gt & 1
                yield from wait("vscales", gt % N, gt // N)
                yield from wait("vfree", g, (gt >> 1) - 1)
                if u < raw_tiles(n, tree):
                    yield from wait("vfull", slot, phase)
                    vtile[g][side].write(gt)
                    rawv[slot].read(gt)
                    vm[gt % N].read(gt)
                    vm[gt % N].readers += 1
                    yield
                    vm[gt % N].readers -= 1
                    B["vempty"][slot].arrive()
                    slot, phase = (0, phase ^ 1) if slot + 1 == ring_v else (slot + 1, phase)
                elif side == 0:
                    vtile[g][0].write(gt)
                    exp[gt & 7].write(gt)
                B["vready"][gt % N].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    def scales(values):
        gt = 0
        for ic in range(len(pieces) + 1):
            n, tree, _ = yield from get(ic)
            if n == 0:
                return
            for u in range(n):
                if gt >= N:
                    yield from wait("vready" if values else "kfree", gt % N, gt // N - 1)
                if u < raw_tiles(n, tree):
                    for x in (vm[gt % N], exp[gt & 7]) if values else (km[gt % N], mids[gt % N]):
                        x.write(gt)
                B["vscales" if values else "kscales"][gt % N].arrive()
                if not values:
                    if u == 0:
                        yield from wait("qready", ic & 1, ic >> 1)
                    if u < raw_tiles(n, tree):
                        factor[gt % (2 * N)].write(gt)
                B["mready"][gt & 7].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    def products():
        gt = gs = ahead = 0

        def qk(ic, half):
            nonlocal ahead
            t, first, last = half
            t += gt
            if first:
                yield from wait("kready", t & 1, t >> 1)
            for x in Q:
                x.readers += 1
            ktile[t & 1][not first].readers += 1
            mids[t % N].readers += 1
            issued.append(("qk", ahead, ic, t, first, last, False))
            ahead += 1

        for ic in range(len(pieces) + 1):
            n, tree, short = yield from get(ic)
            if n == 0:
                return
            halves = _halves(n, tree, short)
            start = gs
            yield from wait("qready", ic & 1, ic >> 1)
            while ahead - start < min(len(halves), N):
                yield from qk(ic, halves[ahead - start])
            for u, (t, first, last) in enumerate(halves):
                t += gt
                if first:
                    yield from wait("vready", t % N, t // N)
                yield from wait("pready", gs % N, gs // N)
                vtile[t & 1][not first].readers += 1
                issued.append(("pv", gs, ic, t, first, last, u < 2))
                gs += 1
                if ahead - start < len(halves):
                    yield from qk(ic, halves[ahead - start])
            gt += n
            B["iempty"][ic & 1].arrive()

    def tensor_core():
        while True:
            if not issued:
                yield
                continue
            kind, gs, ic, t, first, last, fresh = issued[0]      # (in order, one behind the other)
            if kind == "qk":
                S[gs % N].write(gs)
            elif fresh:
                O[gs & 1].write(ic)
            yield
            issued.pop(0)
            if kind == "qk":
                for x in Q:
                    x.read(ic)
                    x.readers -= 1
                ktile[t & 1][not first].read(t)
                mids[t % N].read(t)
                mids[t % N].readers -= 1
                ktile[t & 1][not first].readers -= 1
                B["sfull"][gs % N].arrive()
                if last:
                    B["kfree"][t % N].arrive()
            else:
                S[gs % N].read(gs)
                vtile[t & 1][not first].read(t)
                O[gs & 1].read(ic)
                vtile[t & 1][not first].readers -= 1
                B["pvdone"][gs % N].arrive()
                if last:
                    B["vfree"][t & 1].arrive()

    def softmax_warp(group, w):
        gt = gs = turn = 0
        for ic in range(len(pieces) + 1):
            n, tree, short = yield from get(ic)
            if n == 0:
                return
            first, halves = True, _halves(n, tree, short)
            for u, (t, _, _) in enumerate(halves):
                if gs & 1 != group:
                    gs += 1
                    continue
                g, t = gs % N, t + gt
                yield from wait("mready", t & 7, t >> 3)
                if tree and u == len(halves) - 1:
                    yield from wait("kdone", ic & 1, ic >> 1)
                    yield from wait("vready", t % N, t // N)
                yield from wait("sfull", g, gs // N)
                S[g].read(gs)
                places = (S[g], factor[t % (2 * N)], exp[t & 7])
                for p in places[1:]:
                    p.read(t)
                for p in places:
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
            gt += n
            if len(halves) > 1:
                yield from wait("pvdone", (gs - 2) % N, (gs - 2) // N)
            used = O[:] if len(halves) > 1 else [O[(gs - 1) & 1]]
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

    roles = [copies(), k_tiles(0), k_tiles(1), v_tiles(0), v_tiles(1), scales(False), scales(True), products()] + [softmax_warp(g, w) for g in range(2) for w in range(softmax)]
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


@pytest.mark.parametrize("rings", [(3, 2), (5, 4), (1, 1)])
def test_every_role_ends(rings):
    rng = random.Random(9)
    for _ in range(20):
        pieces = [(rng.choice([1, 1, 2, 3, 4, 7, 12]), rng.random() < 0.5, rng.random() < 0.5) for _ in range(rng.randint(1, 6))]
        _run(pieces, *rings, rng, softmax=rng.choice([1, 4]))


def test_the_kernel_waits_for_what_is_played():
    """The waits of the roles in the source, by barrier."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "tree_attention.cu")).read())
    code = code[code.index("tree_attention_kernel("):code.index("tree_combine_kernel(")]
    cuts = ["if (warp < 8) {", "if (warp < 24) {", "if (warp == 24) {", "if (warp != 26) {", "constexpr uint32_t kIdescS"]
    at = [code.index(x) for x in cuts] + [len(code)]
    waits = [sorted(set(re.findall(r"\bwait\((\w+)", code[a:b]))) for a, b in zip(at, at[1:])]
    assert waits == [["ifull", "kdone", "mready", "pvdone", "sfull", "vready"], ["full", "ifull", "kfree", "scaled", "vfree"],
                     ["iempty", "kempty", "vempty"], ["ifull", "qready", "used"], ["ifull", "kready", "pready", "qready", "vready"]]
    land, done, free = (code.index(x) for x in ("land_after_abort(", "named_bar(2, kDoneThreads)", "tcgen05.dealloc"))
    assert done < land < free and len(re.findall(r"bar_arrive\(2, kDoneThreads\)", code)) == 2
