"""The hand-offs of the latent attention kernel's roles, played through on the host: barriers that count arrivals and know a parity, roles that run in any order, pieces of any
length.  A wait that looks for a phase which its barrier has left behind by two would never end; neither would a circle of roles.  Also what is handed over: nobody writes a place
that somebody still reads."""
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
    """Written by a role for a tile (or piece, or use), read by others of the same."""
    def __init__(self, name):
        self.name, self.of, self.readers = name, None, 0

    def write(self, of):
        assert self.readers == 0, f"{self.name} of {self.of} overwritten while it is read"
        self.of = of

    def read(self, of):
        assert self.of == of, f"{self.name}: {self.of} instead of {of}"


class Meeting:
    """A barrier of a fixed set of threads."""
    def __init__(self, n):
        self.turns = [0] * n

    def at(self, i):
        self.turns[i] += 1
        while min(self.turns) < self.turns[i]:
            yield


FAC, GROUPS = 4, 4


def _run(pieces, K, S_places, rng, warps=1, soft=2, without=()):
    """pieces: tiles of each.  K, S_places: places for keys and scores.  warps: of either set that expands codes; soft: of either half of the softmax.  without: what is left out, to see
    that it is missed."""
    B = {}
    for name, n, count in (("kready", K, warps), ("kfree", K, 1), ("rready", 1, 2 * warps), ("rfree", 1, 1), ("vready", GROUPS, warps), ("vfree", GROUPS, 1), ("fready", FAC, 1),
                           ("ffree", FAC, 2 * soft + 2 * warps), ("sfull", S_places, 1), ("sfree", S_places, 2 * soft), ("pready", 1, 2 * soft), ("odone", 1, 1), ("ifull", 2, 1),
                           ("iempty", 2, 2 * soft + 2 * warps + 3), ("qready", 2, 2 * warps), ("qfree", 1, 1)):
        B[name] = [Barrier(count) for _ in range(n)]
    keys = [[Place(f"keys {i} {w}") for w in range(warps)] for i in range(K)]
    vals = [[Place(f"values {i} {w}") for w in range(warps)] for i in range(GROUPS)]
    rope = [Place(f"rotary {i}") for i in range(2 * warps)]
    q, lim = [Place(f"Q {i}") for i in range(2 * warps)], [[Place(f"limits {i} {j}") for j in range(2 * warps)] for i in range(2)]
    S, fac, item = [Place(f"S {i}") for i in range(S_places)], [Place(f"exponent {i}") for i in range(FAC)], [Place("item 0"), Place("item 1")]
    P, sums = ([[Place(f"{x} {g} {w}") for w in range(soft)] for g in range(2)] for x in ("P", "sums"))
    refs, final, O = [Place("references 0"), Place("references 1")], [Place("last references 0"), Place("last references 1")], Place("O")
    half, both = [Meeting(soft), Meeting(soft)], Meeting(2 * soft)
    queues = {"scores": [], "products": []}       # either thread's, in order

    def wait(bar, i, phase):
        while not B[bar][i].done(phase):
            yield
        yield

    def get(ic):
        yield from wait("ifull", ic & 1, ic >> 1)
        item[ic & 1].read(ic)
        return pieces[ic] if ic < len(pieces) else 0

    def dealer():
        for ic in range(len(pieces) + 1):
            if ic > 1:
                yield from wait("iempty", ic & 1, (ic >> 1) - 1)
            item[ic & 1].write(ic)
            B["ifull"][ic & 1].arrive()
            yield

    def exponents():
        gt = 0
        for ic in range(len(pieces) + 1):
            n = yield from get(ic)
            if n == 0:
                return
            for _ in range(n):
                if gt >= FAC:
                    yield from wait("ffree", gt % FAC, gt // FAC - 1)
                fac[gt % FAC].write(gt)
                B["fready"][gt % FAC].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    def codes(side, w):
        gt, me = 0, 2 * w + side
        for ic in range(len(pieces) + 1):
            n = yield from get(ic)
            if n == 0:
                return
            if ic > 0 and "qfree" not in without:
                yield from wait("qfree", 0, ic - 1)
            q[me].write(ic)
            lim[ic & 1][me].write(ic)
            B["qready"][ic & 1].arrive()
            for _ in range(n):
                yield from wait("fready", gt % FAC, gt // FAC)
                fac[gt % FAC].read(gt)
                B["ffree"][gt % FAC].arrive()
                if gt > 0:
                    yield from wait("rfree", 0, gt - 1)
                rope[me].write(gt)
                B["rready"][0].arrive()
                for g in (side, side + 2):
                    use = gt * GROUPS + g
                    if use >= K:
                        yield from wait("kfree", use % K, use // K - 1)
                    keys[use % K][w].write(use)
                    B["kready"][use % K].arrive()
                    if gt > 0 and "vfree" not in without:
                        yield from wait("vfree", g, gt - 1)
                    vals[g][w].write(gt)
                    B["vready"][g].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    def issue(queue, reads, writes, commits):
        for p, of in reads:
            p.read(of)
            p.readers += 1
        queues[queue].append((reads, writes, commits))

    def scores():
        gt = 0
        for ic in range(len(pieces) + 1):
            n = yield from get(ic)
            if n == 0:
                return
            yield from wait("qready", ic & 1, ic >> 1)
            for u in range(n):
                si = gt % S_places
                if gt >= S_places:
                    yield from wait("sfree", si, gt // S_places - 1)
                yield from wait("rready", 0, gt)
                issue("scores", [(p, gt) for p in rope] + [(p, ic) for p in q], [(S[si], gt)], [("rfree", 0)])
                for g in range(GROUPS):
                    use = gt * GROUPS + g
                    yield from wait("kready", use % K, use // K)
                    last = g == GROUPS - 1
                    issue("scores", [(p, use) for p in keys[use % K]] + [(p, ic) for p in q], [(S[si], gt)],
                          [("kfree", use % K)] + [("sfull", si)] * last + [("qfree", 0)] * (last and u == n - 1))
                gt += 1
            B["iempty"][ic & 1].arrive()

    def products():
        gt = 0
        for ic in range(len(pieces) + 1):
            n = yield from get(ic)
            if n == 0:
                return
            for _ in range(n):
                for g in range(GROUPS):
                    yield from wait("vready", g, gt)
                yield from wait("pready", 0, gt)
                for g in range(GROUPS):
                    issue("products", [(p, gt) for p in vals[g]] + [(p, gt) for x in P for p in x], [(O, ic)], [("vfree", g)] + [("odone", 0)] * (g == GROUPS - 1))
                gt += 1
            B["iempty"][ic & 1].arrive()

    def core(queue):
        while True:
            if not queues[queue]:
                yield
                continue
            reads, writes, commits = queues[queue][0]
            for p, of in writes:
                p.write(of)
            yield
            queues[queue].pop(0)
            for p, of in reads:
                p.read(of)
                p.readers -= 1
            for bar, i in commits:
                B[bar][i].arrive()

    def softmax(h, w):
        gt, me = 0, 2 * w + h
        for ic in range(len(pieces) + 1):
            n = yield from get(ic)
            if n == 0:
                return
            yield from wait("qready", ic & 1, ic >> 1)
            if w == 0:
                refs[h].write(ic)
            if "meeting" not in without:
                yield from both.at(me)
            for u in range(n):
                yield from wait("fready", gt % FAC, gt // FAC)
                yield from wait("sfull", gt % S_places, gt // S_places)
                used = [(S[gt % S_places], gt), (fac[gt % FAC], gt), (refs[h], ic)] + [(p, ic) for p in lim[ic & 1]]
                for p, of in used:
                    p.read(of)
                    p.readers += 1
                yield
                raised = u == 0 or (gt * 7 + ic + h) % 5 == 0       # references are set anew (the same for all of a half)
                if raised:
                    used[2][0].readers -= 1
                    yield from half[h].at(w)
                    if w == 0:
                        refs[h].write(ic)
                    yield from half[h].at(w)
                    refs[h].readers += 1
                    if u > 0:
                        yield from wait("odone", 0, gt - 1)
                        O.read(ic)
                        assert not queues["products"], "rescaled while products are added"
                yield from half[h].at(w)
                for p, _ in used:
                    p.readers -= 1
                if gt > 0:
                    yield from wait("odone", 0, gt - 1)
                P[h][w].write(gt)
                for bar, i in (("pready", 0), ("sfree", gt % S_places), ("ffree", gt % FAC)):
                    B[bar][i].arrive()
                gt += 1
            sums[h][w].write(ic)
            if w == 0:
                refs[h].read(ic)
                final[h].write(ic)
            yield from both.at(me)
            yield from wait("odone", 0, gt - 1)
            used = [(O, ic)] + [(p, ic) for x in sums for p in x] + [(p, ic) for p in final]
            for p, of in used:
                p.read(of)
                p.readers += 1
            for _ in range(rng.choice([1, 1, 4, 40])):
                yield
            for p, of in used:
                p.read(of)
                p.readers -= 1
            B["iempty"][ic & 1].arrive()

    roles = [dealer(), exponents(), scores(), products()] + [codes(s, w) for s in range(2) for w in range(warps)] + [softmax(h, w) for h in range(2) for w in range(soft)]
    cores = [core("scores"), core("products")]
    speed, core_speed, idle = [rng.choice([1, 1, 1, 3, 30, 200]) for _ in roles], [rng.choice([1, 3, 30]) for _ in cores], 0
    state = lambda: ([(b.phase, b.left) for bs in B.values() for b in bs], [len(x) for x in queues.values()], [list(m.turns) for m in (*half, both)])
    while roles:
        before = state()
        for i in rng.sample(range(len(roles)), len(roles)):
            if rng.random() * speed[i] < 1:
                try:
                    next(roles[i])
                except StopIteration:
                    roles[i] = None
        for c, s in zip(cores, core_speed):
            if rng.random() * s < 1:
                next(c)
        keep = [i for i, r in enumerate(roles) if r is not None]
        ended = len(keep) < len(roles)
        roles, speed = [roles[i] for i in keep], [speed[i] for i in keep]
        idle = 0 if ended or before != state() else idle + 1
        assert idle < 20000, "nobody moves"
    assert not any(queues.values())      # (tensor memory is given back behind the last product)


def _pieces(rng):
    return [rng.choice([1, 1, 1, 2, 3, 5, 9]) for _ in range(rng.randint(1, 7))]


@pytest.mark.parametrize("K,S", [(2, 1), (4, 2)])
def test_every_role_ends(K, S):
    rng = random.Random(K)
    for _ in range(25):
        _run(_pieces(rng), K, S, rng, warps=rng.choice([1, 2]), soft=rng.choice([1, 2, 4]))


@pytest.mark.parametrize("without", ["meeting", "vfree", "qfree"])
def test_what_is_left_out_is_missed(without):
    rng = random.Random(1)
    with pytest.raises(AssertionError, match="overwritten|instead of"):
        for _ in range(300):
            _run(_pieces(rng), 4, 2, rng, without=(without,))


def test_the_kernel_waits_for_what_is_played():
    """Waits, and barriers' arrivals, of the roles in the source."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "latent_attention.cu")).read())
    code = code[code.index(") latent_attention_kernel("):code.index("latent_join_kernel(")]
    cuts = ["if (warp < 8) {", "if (warp < 24) {", "if (warp < 26) {", "if (warp == 27) {"]
    at = [code.index(x) for x in cuts]
    at += [code.index("return;\n  }\n", at[-1]), len(code)]
    waits = [sorted(set(re.findall(r"\bwait\((\w+)", code[a:b]))) for a, b in zip(at, at[1:])]
    assert waits == [["fready", "ifull", "odone", "qready", "sfull"], ["fready", "ifull", "kfree", "qfree", "rfree", "vfree"],
                     ["ifull", "kready", "pready", "qready", "rready", "sfree", "vready"], ["iempty"], ["ffree", "ifull"]]
    gives = [sorted(set(re.findall(r"\b(?:mbar_arrive|tc_commit)\((\w+)", code[a:b]))) for a, b in zip(at, at[1:])]
    assert gives == [["ffree", "iempty", "pready", "sfree"], ["ffree", "iempty", "kready", "qready", "rready", "vready"],
                     ["iempty", "kfree", "odone", "qfree", "rfree", "sfull", "vfree"], ["ifull"], ["fready", "iempty"]]
    assert len(re.findall(r"named_bar\(3, 256\)", code)) == 2 and len(re.findall(r"bar_arrive\(4, kDoneThreads\)", code)) == 3
    done, land, free = (code.index(x) for x in ("named_bar(4, kDoneThreads)", "land_after_abort(", "tcgen05.dealloc"))
    assert done < land < free
