"""What the warps with codes of the tree attention kernel tell one another and the other roles through shared memory, played through on the host: the queries' maxima
and sums, the rows' factors, the factor word of a piece, the notes beside the nodes' keys and values.  Nobody writes a place that somebody still reads, and who
reads finds what was written for it.  Also with waits that give up: every role still ends.  (The tiles, scores and sums themselves: test_tree_handoffs.  A tile is one half here.)"""
import os
import random
import re

import pytest

from test_tree_handoffs import CSRC, Barrier, Place

W = 16      # warps with codes: 8 + i; warp i & 3 is a row's part of tensor memory, i >> 2 the quarter of its channels; i & 2: values


class Abandoned:
    """A place as it is once a wait has given up: anything may be in it."""
    readers = 0

    def write(self, what):
        pass

    def read(self, what):
        pass


def _run(pieces, rng, give_up=None):
    """pieces: (tiles, whether the last is the nodes', whether rows need a power of two of their own; 2: and none sees a node).  give_up: the number of waits after which all waits for
    data end at once."""
    place = (lambda name: Abandoned()) if give_up is not None else Place
    B = {name: [Barrier(count) for _ in range(n)] for name, n, count in
         (("ifull", 2, 1), ("iempty", 2, W + 4), ("qready", 2, W), ("kready", 2, 8), ("vready", 3, 8), ("kfree", 3, 1), ("vfree", 2, 1), ("pready", 3, 1), ("mready", 8, 2), ("kscales", 3, 1), ("vscales", 3, 1), ("sfull", 3, 1))}
    maxima, Q = [place(f"maxima {i}") for i in range(W)], [place(f"Q {i}") for i in range(W)]
    sums = [place(f"sums {i}") for i in range(W)]                      # of warp i & 3's rows, a word for each quarter
    factor = [[place(f"factor {q} {i}") for i in range(4)] for q in range(2)]
    word = [place("word 0"), place("word 1")]
    notes = {kind: [[place(f"{kind} notes {g} {i}") for i in range(8)] for g in range(2)] for kind in "kv"}
    met = {}
    waits = 0

    def wait(bar, i, parity, item=False):
        nonlocal waits
        waits += 1
        while not B[bar][i].done(parity) and (item or give_up is None or waits < give_up):
            yield
        yield

    def meet(name, i, n):
        count = met.setdefault(name, [0] * n)
        count[i] += 1
        while min(count) < count[i]:
            yield

    def read(places, what):
        for p in places:
            p.read(what)
            p.readers += 1
        yield
        for p in places:
            p.readers -= 1

    def get(ic):
        yield from wait("ifull", ic & 1, ic >> 1, item=True)
        return pieces[ic] if ic < len(pieces) else (0, False, False)

    def copies():
        for ic in range(len(pieces) + 1):
            yield from wait("iempty", ic & 1, (ic >> 1) - 1, item=True)
            B["ifull"][ic & 1].arrive()

    def codes(i):
        values, w8, gt = bool(i & 2), (i >> 2) * 2 + (i & 1), 0
        own = [(i & 3) + 4 * k for k in range(4)]                      # the four warps of this warp's rows
        for ic in range(len(pieces) + 1):
            n, tree, apart = yield from get(ic)
            if n == 0:
                return
            # queries
            maxima[i].write(ic)
            yield from meet("1", i, W)
            yield from read(maxima, ic)
            if gt > 0:
                yield from wait("kfree", (gt - 1) % 3, (gt - 1) // 3)
            if apart:
                sums[i].write((ic, "largest"))
                yield from meet("1", i, W)
                yield from read([sums[k] for k in own], (ic, "largest"))
                if apart == 2:                                         # (none sees a node: the smallest row)
                    maxima[i].write((ic, "smallest"))
                    yield from meet("1", i, W)
                    yield from read(maxima, (ic, "smallest"))
                yield from meet("1", i, W)
            if i == 0:
                word[ic & 1].write(ic)
            Q[i].write(ic)
            sums[i].write((ic, "sum"))
            yield from meet("1", i, W)
            if i < 4:
                yield from read([sums[k] for k in own], (ic, "sum"))
                for k in own:
                    sums[k].write((ic, "product"))
                factor[ic & 1][i].write(ic)
            B["qready"][ic & 1].arrive()
            # tiles
            for u in range(n):
                g, kind = gt & 1, "v" if values else "k"
                yield from wait(kind + "scales", gt % 3, gt // 3)
                if values:
                    yield from wait("vfree", g, (gt >> 1) - 1)
                elif gt > 1:
                    yield from wait("kfree", (gt - 2) % 3, (gt - 2) // 3)
                mine = notes[kind][g]
                if tree and u == n - 1:
                    mine[w8].write(gt)
                    yield from meet("3" if values else "8", w8, 8)
                    if not values:
                        yield from read([mine[(w8 & 1) + 2 * k] for k in range(4)], gt)
                else:
                    mine[w8].write(None)                               # (the tile's rows 64 to 127)
                B["vready" if values else "kready"][gt % 3 if values else g].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    def scales(values):
        gt = 0
        for ic in range(len(pieces) + 1):
            n, _, _ = yield from get(ic)
            if n == 0:
                return
            for u in range(n):
                if gt >= 3:
                    yield from wait("vready" if values else "kfree", gt % 3, gt // 3 - 1)
                B["vscales" if values else "kscales"][gt % 3].arrive()
                if not values and u == 0:
                    yield from wait("qready", ic & 1, ic >> 1)
                    yield from read([word[ic & 1]], ic)
                B["mready"][gt & 7].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    def products():
        gt = 0
        for ic in range(len(pieces) + 1):
            n, _, _ = yield from get(ic)
            if n == 0:
                return
            yield from wait("qready", ic & 1, ic >> 1)
            done = 0
            for u in range(n):
                while done < min(n, u + 2):                            # (scores a tile ahead of the values)
                    t = gt + done
                    yield from wait("kready", t & 1, t >> 1)
                    for p in Q:
                        p.readers += 1
                    # the sums, and the factors as the other half of their rows, which any power of two may be
                    yield from read(sums, (ic, "product"))
                    for p in Q:
                        p.read(ic)
                        p.readers -= 1
                    B["sfull"][t % 3].arrive()
                    B["kfree"][t % 3].arrive()
                    done += 1
                t = gt + u
                yield from wait("vready", t % 3, t // 3)
                yield from wait("pready", t % 3, t // 3)
                B["vfree"][t & 1].arrive()
            gt += n
            B["iempty"][ic & 1].arrive()

    def softmax():
        gt = 0
        for ic in range(len(pieces) + 1):
            n, tree, _ = yield from get(ic)
            if n == 0:
                return
            for u in range(n):
                yield from wait("mready", gt & 7, gt >> 3)
                yield from wait("sfull", gt % 3, gt // 3)
                yield from read(factor[ic & 1], ic)
                if tree and u == n - 1:
                    yield from wait("vready", gt % 3, gt // 3)
                    yield from read(notes["v"][gt & 1], gt)
                B["pready"][gt % 3].arrive()
                gt += 1
            B["iempty"][ic & 1].arrive()

    roles = [copies(), scales(False), scales(True), products(), softmax()] + [codes(i) for i in range(W)]
    speed = [rng.choice([1, 1, 1, 3, 30]) for _ in roles]
    idle = 0
    while roles:
        before = [(b.phase, b.left) for bs in B.values() for b in bs], {k: list(v) for k, v in met.items()}
        for i in rng.sample(range(len(roles)), len(roles)):
            if rng.random() * speed[i] < 1:
                try:
                    next(roles[i])
                except StopIteration:
                    roles[i] = None
        keep = [i for i, r in enumerate(roles) if r is not None]
        roles, speed = [roles[i] for i in keep], [speed[i] for i in keep]
        idle = idle + 1 if before == ([(b.phase, b.left) for bs in B.values() for b in bs], {k: list(v) for k, v in met.items()}) else 0
        assert idle < 5000, "nobody moves"


def _pieces(rng):
    return [(rng.choice([1, 1, 2, 3, 6]), rng.random() < 0.7, rng.choice([0, 0, 1, 2])) for _ in range(rng.randint(1, 6))]


@pytest.mark.parametrize("seed", range(4))
def test_exchanges(seed):
    rng = random.Random(seed)
    for _ in range(8):
        _run(_pieces(rng), rng)


@pytest.mark.parametrize("seed", range(4))
def test_every_role_ends_when_a_wait_gives_up(seed):
    rng = random.Random(100 + seed)
    for _ in range(8):
        _run(_pieces(rng), rng, give_up=rng.choice([0, 5, 40, 150]))


def test_the_kernel_exchanges_what_is_played():
    """The barriers of the warps with codes in the source, in order, and how often each is met."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "tree_attention.cu")).read())
    body = code[code.index("if (warp < 24) {"):code.index("if (warp == 24) {")]
    assert re.findall(r"named_bar\((\d+), \d+\)|\b(row_maxima|largest_of_8)\(", body) == [
        ("", "row_maxima"), ("1", ""), ("", "row_maxima"), ("1", ""), ("1", ""), ("", "largest_of_8"), ("8", "")]
    for name, bar in (("RowMaxima row_maxima(", "named_bar(1, 512)"), ("uint32_t largest_of_8(", "named_bar(3, 256)")):
        f = code[code.index(name):]
        f = f[:f.index("\n}")]
        assert f.count("named_bar(") == 1 and bar in f
        assert f.index("volatile uint") < f.index("named_bar(") < f.index("lds64(")      # written, met, read
    # (the sums are free from the previous piece's last product on)
    assert body.index("wait(kfree + ms.before(1)") < body.index("sts32(sums + quarter * 4u, mine)")
