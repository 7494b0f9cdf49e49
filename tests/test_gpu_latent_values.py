"""Attention over quantised latents against 64 bits whose values are rounded as the kernel rounds them (see latent_rounded.py, also for the bounds), for queries that look for
single tokens: the ends of a sequence, of a mask and of tiles among them.  tests/test_latent_rounded.py shows what those bounds turn away."""
import pytest
import torch

import latent_rounded as ref
import paper_2607_01831_b200 as lynx
import test_gpu_latent_attention as base
import test_gpu_latent_serving as serving

pytestmark = pytest.mark.gpu


def _held(cache, b, anchor):
    """Rounded values [L][512] and rotary keys [L][64] of sequence b."""
    t = torch.arange(cache.lens[b])
    blk, off = cache.table[b, t // cache.bt].long().cuda(), (t % cache.bt).cuda()
    return ref.rounded(lynx.recombine(cache.planes)[0][blk, :, off], cache.planes.meta[blk, :, off], anchor), cache.pages[blk, off].double()


def _pointed(cache, n, H, causal, a, seed):
    """Queries [B][n][H][512] and [B][n][H][64], views of one tensor."""
    g = torch.Generator().manual_seed(seed)
    both = torch.zeros(len(cache.lens), n, H, 576, dtype=torch.bfloat16)
    for b, L in enumerate(cache.lens):
        if L:
            counts = [max(0, L - n + j + 1) if causal else L for j in range(n)]
            both[b, ..., :512], both[b, ..., 512:] = ref.pointed_queries(*_held(cache, b, False), counts, H, a, g)
    both = both.cuda()
    return both[..., :512], both[..., 512:]


def check(cache, q, qr, out, lse, causal, anchor, scale=0.0, only=None, positions=None):
    B, n, H, _ = q.shape
    a = scale or 192 ** -0.5
    step = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    tiles = [-(-x // 128) for x in cache.lens]
    per_cta = min(max(max(tiles), 1), sum(tiles) * -(-n * H // 64) // 125 + 2)
    for b in range(B) if only is None else only:
        L = cache.lens[b]
        v, keys = _held(cache, b, anchor) if L else (None, None)
        for j in range(n) if positions is None else positions:
            count = max(0, L - n + j + 1) if causal else L
            gl = None if lse is None else lse[b, j]
            if count == 0:
                assert not out[b, j].any() and (gl is None or (gl == -float("inf")).all())
                continue
            far = ref.worst(out[b, j], gl, v[:count], keys[:count], q[b, j], qr[b, j], a, step, per_cta)
            assert far <= 1.0, (b, j, far)


@pytest.mark.parametrize("lens", base.LENS)
@pytest.mark.parametrize("n,H", [(1, 1), (1, 16), (1, 20), (1, 64), (1, 128), (3, 16), (5, 40), (64, 2)])
@pytest.mark.parametrize("anchor", [False, True])
def test_lengths_rows_and_planes(lens, n, H, anchor):
    cache = base.Cache(lens, 16 if n < 5 else 32, H, seed=sum(lens) + H, wide=n)
    some = None if n < 64 else (0, 1, 31, 62, 63)
    for causal in (True, False):
        q, qr = _pointed(cache, n, H, causal, 192 ** -0.5, n + H)
        for out in (None, torch.full(q.shape, 7.0, device="cuda")):
            out, lse = base._run(cache, q, qr, causal, anchor, out=out)
            check(cache, q, qr, out, lse, causal, anchor, positions=some)


@pytest.mark.parametrize("lens,n,H,anchor", [((20000,), 1, 16, True), ((9000, 20011, 333), 4, 32, False), ((7000,) * 5, 1, 128, False), ((60001,), 1, 64, False),
                                             ((30000, 2, 9999), 1, 32, True)])
def test_long_contexts_in_many_parts(lens, n, H, anchor):
    cache = base.Cache(lens, 64, H, seed=9, junk=False)
    q, qr = _pointed(cache, n, H, True, 192 ** -0.5, 2)
    out, lse = base._run(cache, q, qr, True, anchor, out=torch.empty(q.shape, device="cuda"))
    check(cache, q, qr, out, lse, True, anchor)


@pytest.mark.parametrize("n,H", [(1, 16), (1, 32), (2, 64)])
def test_many_sequences(n, H):
    lens = [i * 37 % 611 for i in range(200)]
    cache = base.Cache(lens, 16, H, seed=5)
    q, qr = _pointed(cache, n, H, True, 192 ** -0.5, 3)
    out, lse = base._run(cache, q, qr)
    check(cache, q, qr, out, lse, True, False, only=range(0, 200, 7))


@pytest.mark.parametrize("H", [16, 32, 64, 100])
@pytest.mark.parametrize("anchor", [False, True])
def test_all_channels_at_once(H, anchor):
    """Queries without zeros."""
    cache = base.Cache((900, 77), 16, H, seed=31)
    q, qr = base._queries(2, 1, H, seed=32)
    out, lse = base._run(cache, q, qr, True, anchor, out=torch.empty(q.shape, device="cuda"))
    check(cache, q, qr, out, lse, True, anchor)


@pytest.mark.parametrize("spread,scale", [(1e-20, 0.0), (300.0, 0.02), (1e10, 0.5)])
@pytest.mark.parametrize("H", [16, 64])
def test_scales_of_any_size(spread, scale, H):
    cache = base.Cache((700, 33), 16, H, seed=4, spread=spread)
    cache.pages *= spread
    q, qr = _pointed(cache, 1, H, True, scale or 192 ** -0.5, 5)
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"), scale=scale)
    check(cache, q, qr, out, lse, True, False, scale=scale)


def test_a_chunk_of_a_prompt():
    """64 positions of 128 heads: 128 row tiles a sequence."""
    cache = base.Cache((300, 64), 32, 128, seed=33)
    q, qr = _pointed(cache, 64, 128, True, 192 ** -0.5, 34)
    out, lse = base._run(cache, q, qr)
    check(cache, q, qr, out, lse, True, False, positions=(0, 1, 40, 63))


@pytest.mark.parametrize("at", [0, 1500, 4000])
@pytest.mark.parametrize("H", [16, 40])
def test_references_that_are_raised(at, H):
    """Scores that grow along the context by the rotary keys' first channel, and one token far above the rest."""
    cache = base.Cache((4001,), 16, H, seed=6)
    t = torch.arange(4001)
    blk, off = cache.table[0, t // 16].long().cuda(), (t % 16).cuda()
    q, qr = _pointed(cache, 2, H, True, 192 ** -0.5, 7)
    cache.pages[blk, off, 0] = torch.linspace(0, 3, 4001).to(torch.bfloat16).cuda()
    qr[..., 0] = 60.0 * (1 + torch.arange(H, device="cuda") % 3)
    cache.pages[blk[at], off[at], 1] = 30.0
    qr[..., 1] = 12.0
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    check(cache, q, qr, out, lse, True, False)


@pytest.mark.parametrize("zeros", [(0, 128), (128, 256), (100, 400), (0, 700)])
def test_tiles_of_zeros(zeros):
    cache = base.Cache((700,), 16, 20, seed=29)
    t = torch.arange(*zeros)
    q, qr = _pointed(cache, 2, 20, True, 192 ** -0.5, 30)
    cache.planes.meta[cache.table[0, t // 16].long().cuda(), :, (t % 16).cuda()] = 0.0
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    check(cache, q, qr, out, lse, True, False)


def test_tokens_of_very_different_sizes():
    """Within a tile: a token of tiny values that takes most of the weight, one of zeros, outliers in a row; scales that are subnormal in FP16."""
    cache = base.Cache((2000,), 16, 16, seed=8, channels=False)
    t = torch.arange(2000)
    blk, off = cache.table[0, t // 16].long().cuda(), (t % 16).cuda()
    cache.planes.meta[blk[5], :, off[5]] *= 2.0 ** -30
    cache.planes.meta[blk[300], :, off[300]] = 0.0
    cache.planes.meta[blk[777], 1, off[777]] *= 2.0 ** 7
    for i, size in ((900, -12), (901, -18), (902, -22), (903, -25), (904, -28)):
        cache.planes.meta[blk[i], :, off[i]] *= 2.0 ** size
    q, qr = base._queries(1, 1, 16, seed=9)
    q, qr = q * 0.01, qr.abs()
    for h, i in enumerate((5, 300, 777, 900, 901, 902, 903, 904)):
        cache.pages[blk[i], off[i], 8 * h:8 * h + 8] = 4.0
        qr[:, :, h::8, 8 * h:8 * h + 8] = 8.0
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    check(cache, q, qr, out, lse, True, False)


def test_replayed_for_other_lengths():
    cache = base.Cache((600, 200), 16, 16, seed=16, wide=4)
    q, qr = _pointed(cache, 1, 16, True, 192 ** -0.5, 17)
    ws = lynx.make_latent_workspace(cache.geo, 2, 1, "cuda")
    base._run(cache, q, qr, ws=ws)
    graph, out = torch.cuda.CUDAGraph(), torch.empty(2, 1, 16, 512, device="cuda")
    with torch.cuda.graph(graph):
        lynx.latent_attention(cache.geo, q, qr, cache.planes, cache.pages, cache.d_table, cache.d_lens, ws, out=out)
    for lens in ((600, 200), (17, 130), (1, 0)):
        cache.lens = list(lens)
        cache.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check(cache, q, qr, out, None, True, False)


def test_what_a_server_attends_to():
    """The example's chunks of prompts and its decode steps, in shuffled blocks of a pool."""
    class Server(serving._Watched):
        def check(self):
            q, qr, table, lens, out = self.seen
            check(serving._Held(self, table, lens), q, qr, out, None, True, False, positions=range(0, q.shape[1], 9))

    server = Server(serving.example.Layer(vocab=256, dim=256, heads=8), 3, 26, 448)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(256, (n,), generator=g).cuda() for n in (90, 300, 64, 200)]
    real = server.step

    def step():
        real()
        server.check()

    server.step = step
    got, _ = serving.example.serve(server, prompts, 12)
    assert all(len(x) == 12 for x in got)
