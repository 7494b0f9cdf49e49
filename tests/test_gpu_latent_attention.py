"""Attention over quantised latents against 64 bits, on the planes' exact values.

Bounds, with U = 2^-11, FP16's eps / 2, and 2^-24 of FP32.
Values: a row's scale and middle (zero + 128 scale) are rounded to FP16, then middle + scale (code - 128): U (|middle| + |code - 128| scale) + U |value|, at
most 2 U M with M = |middle| + 128 scale, which no channel of the row exceeds.
Scores: |ds| <= a sum_d |q_d| (2 U M_d) over the latent's channels (queries are exact), plus the accumulation of 576 terms, truncating: 2^-23 * 576 < 2^-13 of a sum of
|q| M and |q_r k_r|, and the few FP32 operations behind it.  With D the largest of that over the tokens that a row sees, a weight is off by a factor e^+-D, and weight over
sum by 2 D (1 + D) at most.
Outputs: weights are rounded (U), values as above, the second product's sums truncate (2^-13 of sum p |v|, as above, per 128 tokens, and FP32 from tile to tile: tokens / 128 *
2^-24), so |out - want| <= (2 D + 2 D^2 + 3 U + 2^-12 + tokens 2^-31) sum p M, and half a step of the output's type.  Weights below FP16's range are 2^-28 of the row's largest
2^e p, an absolute 2^-25 of it: covered by tokens * 2^-26 max M.
Log-sum-exps: D, and 2^-20 of 1 + |lse|."""
import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu
U = 2.0 ** -11


def _gen(seed):
    return torch.Generator().manual_seed(seed)


class Cache:
    """A pool of quantised latents and rotary keys in shuffled blocks; what no sequence holds is no number."""

    def __init__(self, lens, bt, Hq, seed=0, spread=1.0, channels=True, wide=0, junk=True):
        g = _gen(seed)
        self.lens, self.bt, B = list(lens), bt, len(lens)
        need = [-(-n // bt) for n in lens]
        self.nb = sum(need) + 3
        self.table = torch.full((B, max(1, max(need)) + wide), -9 if junk else 0, dtype=torch.int32)
        ids = torch.randperm(self.nb, generator=g).to(torch.int32)
        for b, n in enumerate(need):
            self.table[b, :n] = ids[sum(need[:b]):sum(need[:b]) + n]
        x = torch.randn(self.nb, 4, bt, 128, generator=g) * spread
        if channels:
            x *= torch.exp(0.7 * torch.randn(4, 1, 128, generator=g))
        self.planes = lynx.split_quantize(x.to(torch.bfloat16).cuda())
        self.pages = torch.randn(self.nb, bt, 64, generator=g).to(torch.bfloat16).cuda()
        if junk:       # rows behind a sequence's end, and blocks of none
            dead = torch.ones(self.nb * bt, dtype=torch.bool)
            for b, n in enumerate(lens):
                t = torch.arange(n)
                dead[self.table[b, t // bt].long() * bt + t % bt] = False
            dead = dead.view(self.nb, bt).cuda()
            self.planes.meta[dead[:, None].expand(self.nb, 4, bt)] = float("nan")
            self.pages[dead] = float("nan")
        self.geo = lynx.Geometry(Hq, 4, bt, self.nb, self.table.shape[1])
        self.d_table, self.d_lens = self.table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()

    def rows(self, b, anchor):
        """float64 latents [tokens][512], the most that a channel of their rows can be, and rotary keys [tokens][64] of sequence b, on the GPU."""
        t = torch.arange(self.lens[b])
        blk, off = self.table[b, t // self.bt].long().cuda(), (t % self.bt).cuda()
        code = lynx.recombine(self.planes)[0][blk, :, off].double()
        if anchor:
            code = torch.floor(code / 16) * 16 + 8
        meta = self.planes.meta[blk, :, off].double()
        size = (meta[..., 1:] + 128 * meta[..., :1]).abs() + 128 * meta[..., :1]
        return (meta[..., 1:] + meta[..., :1] * code).flatten(1), size.expand(-1, -1, 128).flatten(1), self.pages[blk, off].double()


def _queries(B, n, H, seed, spread=1.0):
    g = _gen(seed)
    q = (torch.randn(B, n, H, 576, generator=g) * spread).to(torch.bfloat16).cuda()
    return q[..., :512], q[..., 512:]


def _check(cache, q, qr, out, lse, causal, anchor, scale=0.0, skip=()):
    B, n, H, _ = q.shape
    a = scale or 192 ** -0.5
    step = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    for b, L in enumerate(cache.lens):
        if b in skip:
            continue
        latents, sizes, keys = cache.rows(b, anchor)
        for j in range(n):
            count = max(0, L - n + j + 1) if causal else L
            got, gl = out[b, j].double(), None if lse is None else lse[b, j].double()
            if count == 0:
                assert (got == 0).all() and (gl is None or (gl == -float("inf")).all())
                continue
            v, size, x, y = latents[:count], sizes[:count], q[b, j].double(), qr[b, j].double()
            s = a * (x @ v.T + y @ keys[:count].T)
            w = s.softmax(1)
            want = w @ v
            D = a * ((2 * U + 2.0 ** -13) * (x.abs() @ size.T) + 2.0 ** -13 * (y.abs() @ keys[:count].abs().T)).amax(1, keepdim=True)
            bound = (2 * D + 2 * D * D + 3 * U + 2.0 ** -12 + count * 2.0 ** -31) * (w @ size) + count * 2.0 ** -26 * size.max() + step * want.abs()
            assert ((got - want).abs() <= bound).all(), (b, j, float(((got - want).abs() / bound).max()))
            if gl is not None:
                l = s.logsumexp(1)
                assert ((gl - l).abs() <= D[:, 0] + 2.0 ** -20 * (1 + l.abs())).all()


def _run(cache, q, qr, causal=True, anchor=False, out=None, ws=None, scale=0.0):
    B, n, H, _ = q.shape
    ws = lynx.make_latent_workspace(cache.geo, B, n, "cuda") if ws is None else ws
    lse = torch.full((B, n, H), 7.0, device="cuda")
    out = lynx.latent_attention(cache.geo, q, qr, cache.planes, cache.pages, cache.d_table, cache.d_lens, ws, causal=causal, anchor_only=anchor, lse=lse, out=out,
                                softmax_scale=scale)
    lynx.check(ws)
    return out, lse


LENS = [(1,), (16,), (300,), (128, 129, 0, 127), (1000, 3, 2500), (40, 700, 1, 0, 260, 130, 128, 5, 900)]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("n,H", [(1, 1), (1, 16), (1, 20), (1, 64), (1, 128), (3, 16), (5, 40), (64, 2)])
@pytest.mark.parametrize("anchor", [False, True])
def test_lengths_rows_and_planes(lens, n, H, anchor):
    cache = Cache(lens, 16 if n < 5 else 32, H, seed=sum(lens) + H, wide=n)
    q, qr = _queries(len(lens), n, H, seed=n + H)
    for causal in (True, False):
        out, lse = _run(cache, q, qr, causal, anchor)
        assert out.dtype == torch.bfloat16
        _check(cache, q, qr, out, lse, causal, anchor)


@pytest.mark.parametrize("lens,n,H", [((20000,), 1, 16), ((9000, 20011, 333), 4, 32), ((7000,) * 5, 1, 128), ((131072,), 1, 64)])
def test_long_contexts_in_many_parts(lens, n, H):
    cache = Cache(lens, 64, H, seed=9, junk=False)
    q, qr = _queries(len(lens), n, H, seed=2)
    out, lse = _run(cache, q, qr, True, False, out=torch.empty(q.shape, device="cuda"))
    _check(cache, q, qr, out, lse, True, False)
    again, _ = _run(cache, q, qr, True, False, out=torch.empty(q.shape, device="cuda"))
    assert torch.equal(out, again)


def test_many_sequences():
    lens = [i * 37 % 611 for i in range(200)]
    cache = Cache(lens, 16, 16, seed=5)
    q, qr = _queries(200, 1, 16, seed=3)
    out, lse = _run(cache, q, qr)
    _check(cache, q, qr, out, lse, True, False)


@pytest.mark.parametrize("H,n", [(16, 1), (32, 1), (64, 2)])
def test_many_pieces_of_one_tile(H, n):
    """Each CTA takes several pieces, one behind the other: outputs of one are written while the next one's tile is under way."""
    lens = [i * 53 % 129 for i in range(1100)]
    cache = Cache(lens, 16, H, seed=15, wide=9)
    q, qr = _queries(1100, n, H, seed=16)
    out, lse = _run(cache, q, qr)
    some = set(range(0, 1100, 7))
    _check(cache, q, qr, out, lse, True, False, skip=set(range(1100)) - some)
    for _ in range(5):
        again, l2 = _run(cache, q, qr)
        assert torch.equal(again, out) and torch.equal(l2, lse)


@pytest.mark.parametrize("spread,qs", [(1e-20, 1.0), (1e-3, 100.0), (300.0, 0.01), (1e15, 1e-15), (1.0, 8.0), (1.0, 1e-30)])
@pytest.mark.parametrize("H", [16, 64])
def test_scales_of_any_size(spread, qs, H):
    cache = Cache((700, 33), 16, H, seed=4, spread=spread)
    q, qr = _queries(2, 1, H, seed=5, spread=qs)
    if qs > 1:
        qr = (qr.float() / qs).to(torch.bfloat16)
    out, lse = _run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    _check(cache, q, qr, out, lse, True, False)


@pytest.mark.parametrize("at", [0, 100, 1500, 4000])
@pytest.mark.parametrize("H", [16, 40])
def test_a_dominating_token_raises_the_references(at, H):
    """Scores that grow along the context, and one token far above the rest: early, in the middle, at the end."""
    cache = Cache((4001,), 16, H, seed=6)
    q, qr = _queries(1, 2, H, seed=7)
    t = torch.arange(4001)
    blk, off = cache.table[0, t // 16].long().cuda(), (t % 16).cuda()
    ramp = torch.linspace(0, 3, 4001).to(torch.bfloat16).cuda()
    cache.pages[blk, off, 0] = ramp
    qr[..., 0] = 60.0 * (1 + torch.arange(H, device="cuda") % 3)
    cache.pages[blk[at], off[at], 1] = 30.0
    qr[..., 1] = 12.0
    out, lse = _run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    _check(cache, q, qr, out, lse, True, False)


def test_tokens_of_very_different_sizes():
    """A token of tiny values that takes most of the weight, tokens of zeros, tokens with outliers."""
    cache = Cache((2000,), 16, 16, seed=8, channels=False)
    t = torch.arange(2000)
    blk, off = cache.table[0, t // 16].long().cuda(), (t % 16).cuda()
    cache.planes.meta[blk[5], :, off[5]] *= 2.0 ** -30
    cache.planes.meta[blk[300], :, off[300]] = 0.0
    cache.planes.meta[blk[777], 1, off[777]] *= 2.0 ** 7
    q, qr = _queries(1, 1, 16, seed=9)
    cache.pages[blk[5], off[5]] = 8.0
    qr.abs_()
    out, lse = _run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    _check(cache, q, qr, out, lse, True, False)


def test_what_is_no_number_spoils_no_other_row():
    cache = Cache((500, 260, 90), 16, 20, seed=10)
    q, qr = _queries(3, 2, 20, seed=11)
    clean, _ = _run(cache, q, qr)
    q, qr = q.clone(), qr.clone()
    bad = torch.zeros(3, 2, 20, dtype=torch.bool)
    for (b, j, h), x, t in (((0, 0, 3), float("nan"), q), ((0, 1, 19), float("inf"), q), ((1, 1, 0), float("nan"), qr), ((2, 0, 7), -float("inf"), qr)):
        t[b, j, h, 9] = x
        bad[b, j, h] = True
    out, lse = _run(cache, q, qr)
    assert torch.equal(out[~bad.cuda()], clean[~bad.cuda()]) and lse[~bad.cuda()].isfinite().all()
    # one in a token: the sequence's rows, the others' stay
    cache.planes.meta[cache.table[1, 3], 2, 4] = float("nan")
    out, _ = _run(cache, q, qr)
    keep = ~bad
    keep[1] = False
    assert torch.equal(out[keep.cuda()], clean[keep.cuda()]) and out[1].isnan().any()


def test_strides_scale_workspaces_and_streams(monkeypatch):
    cache = Cache((333, 40), 16, 16, seed=12)
    q, qr = _queries(2, 3, 16, seed=13)
    ws = lynx.make_latent_workspace(cache.geo, 2, 8, "cuda")        # a larger call's serves
    out, lse = _run(cache, q, qr, ws=ws, scale=0.25)
    _check(cache, q, qr, out, lse, True, False, scale=0.25)
    assert torch.equal(_run(cache, q.contiguous(), qr.contiguous(), ws=ws, scale=0.25)[0], out)
    # 16 bytes of alignment are enough
    shift = lambda t: torch.cat((torch.zeros(16 // t.element_size(), dtype=t.dtype, device="cuda"), t.flatten()))[16 // t.element_size():].view(t.shape)
    p = cache.planes
    moved = lynx.Planes(shift(p.anchor), shift(p.residual), shift(p.meta))
    assert moved.anchor.data_ptr() % 32 == 16
    assert torch.equal(lynx.latent_attention(cache.geo, q, qr, moved, shift(cache.pages), cache.d_table, cache.d_lens, ws, softmax_scale=0.25), out)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        side = lynx.latent_attention(cache.geo, q, qr, p, cache.pages, cache.d_table, cache.d_lens, ws, softmax_scale=0.25)
    st.synchronize()
    assert torch.equal(side, out)
    monkeypatch.setattr(lynx, "_fast_latent_attention", lynx._python_only)
    assert torch.equal(lynx.latent_attention(cache.geo, q, qr, p, cache.pages, cache.d_table, cache.d_lens, ws, softmax_scale=0.25), out)


def test_bad_block_ids_are_reported():
    cache = Cache((300,), 16, 16, seed=14, junk=False)
    q, qr = _queries(1, 1, 16, seed=15)
    ws = lynx.make_latent_workspace(cache.geo, 1, 1, "cuda")
    cache.d_table[0, 5] = cache.nb + 100
    cache.d_table[0, 7] = -3
    lynx.latent_attention(cache.geo, q, qr, cache.planes, cache.pages, cache.d_table, cache.d_lens, ws)
    with pytest.raises(lynx.LynxError, match="block id"):
        lynx.check(ws)
    lynx.check(ws)


def test_captured_and_replayed():
    cache = Cache((600, 200), 16, 16, seed=16, wide=4)
    q, qr = _queries(2, 1, 16, seed=17)
    ws = lynx.make_latent_workspace(cache.geo, 2, 1, "cuda")
    _run(cache, q, qr, ws=ws)
    graph, out = torch.cuda.CUDAGraph(), torch.empty(2, 1, 16, 512, device="cuda")
    with torch.cuda.graph(graph):
        lynx.latent_attention(cache.geo, q, qr, cache.planes, cache.pages, cache.d_table, cache.d_lens, ws, out=out)
    for lens in ((600, 200), (17, 130), (1, 0)):
        cache.lens = list(lens)
        cache.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        _check(cache, q, qr, out, None, True, False)


@pytest.mark.parametrize("bt", [48, 112, 128, 400])
def test_blocks_that_end_inside_a_tile(bt):
    cache = Cache((1000, 130, 47), bt, 20, seed=18)
    q, qr = _queries(3, 2, 20, seed=19)
    out, lse = _run(cache, q, qr)
    _check(cache, q, qr, out, lse, True, False)


def test_lengths_beyond_the_table():
    cache = Cache((320, 64), 16, 16, seed=20, junk=False)
    cache.table[1, 4:] = cache.table[1, :1]      # (20 blocks: any will do)
    cache.d_table = cache.table.cuda()
    q, qr = _queries(2, 1, 16, seed=21)
    cache.d_lens.copy_(torch.tensor([320, 320], dtype=torch.int32))
    want, _ = _run(cache, q, qr)
    cache.d_lens.copy_(torch.tensor([2 ** 31 - 1, 321], dtype=torch.int32))
    assert torch.equal(_run(cache, q, qr)[0], want)
    cache.d_lens.copy_(torch.tensor([-5, 0], dtype=torch.int32))
    out, lse = _run(cache, q, qr)
    assert not out.any() and (lse == -float("inf")).all()


def test_two_graphs_of_one_workspace_and_two_streams():
    caches = [Cache((900, 40), 16, 16, seed=22), Cache((333, 2000), 16, 16, seed=23)]
    queries = [_queries(2, 1, 16, seed=24), _queries(2, 1, 16, seed=25)]
    want = [_run(c, *x)[0] for c, x in zip(caches, queries)]
    ws = lynx.make_latent_workspace(lynx.Geometry(16, 4, 16, 9, 200), 2, 1, "cuda")
    call = lambda i, w, out: lynx.latent_attention(caches[i].geo, *queries[i], caches[i].planes, caches[i].pages, caches[i].d_table, caches[i].d_lens, w, out=out)
    outs, graphs = [torch.empty_like(x) for x in want], [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            call(i, ws, outs[i])
    for _ in range(5):
        for i in (0, 1, 1, 0):
            outs[i].zero_()
            graphs[i].replay()
            assert torch.equal(outs[i], want[i])
    lynx.check(ws)
    # a workspace and a stream each
    streams, spaces = [torch.cuda.Stream(), torch.cuda.Stream()], [lynx.make_latent_workspace(c.geo, 2, 1, "cuda") for c in caches]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                call(i, spaces[i], outs[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    for w in spaces:
        lynx.check(w)


def test_planes_of_more_than_four_gigabytes():
    """Blocks at the end of a pool whose planes' and pages' offsets pass 32 bits: written, read back and attended to as at its beginning."""
    bt, tokens = 16, 200
    nb = (1 << 32) // (4 * bt * 64) + 40000
    rows = (nb, 4, bt)
    big = lynx.Planes(torch.empty(*rows, 64, dtype=torch.uint8, device="cuda"), torch.empty(*rows, 64, dtype=torch.uint8, device="cuda"), torch.empty(*rows, 2, device="cuda"))
    pages = torch.empty(nb, bt, 64, dtype=torch.bfloat16, device="cuda")
    g = _gen(26)
    c, k = (torch.randn(tokens, w, generator=g).to(torch.bfloat16).cuda() for w in (512, 64))
    q, qr = _queries(1, 1, 16, seed=27)
    results = []
    for first in (0, nb - 13):
        geo = lynx.Geometry(16, 4, bt, nb, 13)
        blocks = first + torch.randperm(13, generator=_gen(28)).cuda()
        t = torch.arange(tokens, device="cuda")
        lynx.latent_append(geo, c, k, blocks[t // bt] * bt + t % bt, big, pages)
        table, lens = blocks.to(torch.int32)[None], torch.tensor([tokens], dtype=torch.int32).cuda()
        back = lynx.latent_read(geo, big, pages, table, None, torch.tensor([0, tokens], dtype=torch.int32).cuda(), tokens)
        out = lynx.latent_attention(geo, q, qr, big, pages, table, lens, lynx.make_latent_workspace(geo, 1, 1, "cuda"))
        results.append((*back, out))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    # (half a step of a row's span, and BF16's rounding)
    span = (c.view(-1, 4, 128).amax(2) - c.view(-1, 4, 128).amin(2)).double().repeat_interleave(128, 1)
    assert ((results[1][0].double() - c.double()).abs() <= span * (1 + 2.0 ** -6) / 510 + 2.0 ** -8 * c.double().abs().amax()).all() and torch.equal(results[1][1], k)


@pytest.mark.parametrize("zeros", [(0, 128), (128, 256), (100, 400), (0, 700)])
@pytest.mark.parametrize("H", [16, 64, 100])
def test_tiles_of_zeros(zeros, H):
    """Tokens whose latents are zeros, tiles of them: their rotary keys still take weight."""
    cache = Cache((700,), 16, H, seed=29)
    t = torch.arange(*zeros)
    cache.planes.meta[cache.table[0, t // 16].long().cuda(), :, (t % 16).cuda()] = 0.0
    q, qr = _queries(1, 2, H, seed=30)
    out, lse = _run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    _check(cache, q, qr, out, lse, True, False)
