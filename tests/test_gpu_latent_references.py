"""Attention over quantised latents where tiles have powers of two far apart: what a row's weights are relative to follows its scores, and not the sizes of tokens that it does not
look at.  Against 64 bits and the bounds of latent_rounded.py."""
import pytest
import torch

import latent_rounded as ref
import test_gpu_latent_values as values

pytestmark = pytest.mark.gpu
base = values.base
A = 192 ** -0.5


def _cache(tokens, H, big, seed):
    """big: exponents by token.  Such a token's values are all below zero, as far as 2^big times the others'; nobody looks at it."""
    cache = base.Cache((tokens,), 64, H, seed=seed, junk=False)
    for t, k in big.items():
        blk, off = int(cache.table[0, t // 64]), t % 64
        scale = cache.planes.meta[blk, :, off, 0].clone() * 2.0 ** k
        cache.planes.meta[blk, :, off, 0] = scale
        cache.planes.meta[blk, :, off, 1] = -300 * scale
    return cache


def _queries(cache, n, H, seed):
    v, keys = values._held(cache, 0, False)
    L = cache.lens[0]
    q, qr = ref.pointed_queries(v, keys, [L - n + j + 1 for j in range(n)], H, A, torch.Generator().manual_seed(seed), positive=True)
    both = torch.cat((q, qr), 2)[None].cuda()
    return both[..., :512], both[..., 512:]


# 700 tiles: five a CTA, one behind the other
@pytest.mark.parametrize("k", [6, 10, 20, 30, 60])
@pytest.mark.parametrize("tile", [0, 2, 4])
@pytest.mark.parametrize("n,H", [(1, 16), (2, 16), (1, 64), (1, 100)])
def test_large_tokens_that_take_no_weight(k, tile, n, H):
    big = {128 * t + 77: k for t in range(tile, 700, 5)}
    cache = _cache(128 * 700 - 3, H, big, seed=k)
    q, qr = _queries(cache, n, H, seed=tile)
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    values.check(cache, q, qr, out, lse, True, False)


@pytest.mark.parametrize("pattern", [(0, 40, 0, 20, 0), (50, 30, 10, 30, 0), (0, 0, 60, 3, 60), (5, 4, 3, 2, 1)])
@pytest.mark.parametrize("anchor", [False, True])
def test_sizes_that_come_and_go(pattern, anchor):
    big = {128 * t + 5: pattern[t % 5] for t in range(700) if pattern[t % 5]}
    cache = _cache(128 * 700, 32, big, seed=3)
    q, qr = _queries(cache, 1, 32, seed=4)
    out, lse = base._run(cache, q, qr, True, anchor, out=torch.empty(q.shape, device="cuda"))
    values.check(cache, q, qr, out, lse, True, anchor)


def test_tiles_of_small_values_behind_others():
    """Tiles whose values are all 2^-25 of those in front of them, and where most of the weight is."""
    cache = base.Cache((128 * 700,), 64, 16, seed=5, junk=False)
    t = torch.arange(128 * 700)
    blk, off = cache.table[0, t // 64].long().cuda(), (t % 64).cuda()
    small = (t // 128 % 5 >= 2).cuda()
    cache.planes.meta[blk[small], :, off[small]] *= 2.0 ** -25
    cache.pages[blk[small], off[small], 0] = 4.0
    cache.pages[blk[~small], off[~small], 0] = -4.0
    g = torch.Generator().manual_seed(6)
    both = torch.zeros(1, 1, 16, 576)
    both[..., 512] = 40.0 + torch.arange(16)         # the small tokens' scores are about 25 above the others'
    both[..., 513:520] = torch.randn(16, 7, generator=g)
    both = both.to(torch.bfloat16).cuda()
    q, qr = both[..., :512], both[..., 512:]
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    values.check(cache, q, qr, out, lse, True, False)


@pytest.mark.parametrize("k", [90, 110])
@pytest.mark.parametrize("H", [16, 100])
def test_sizes_too_far_apart(k, H):
    """Beyond 2^64 weights lose bits in the outputs, as documented; sums of weights do not, and nothing overflows."""
    big = {128 * t + 77: k for t in range(1, 700, 3)}
    cache = _cache(128 * 700 - 3, H, big, seed=k)
    q, qr = _queries(cache, 1, H, seed=1)
    out, lse = base._run(cache, q, qr, out=torch.empty(q.shape, device="cuda"))
    v, keys = values._held(cache, 0, False)
    want, l, w = ref.attention(v, keys, q[0, 0], qr[0, 0], A)
    _, bound = ref.bounds(v, keys, q[0, 0], qr[0, 0], A, want, l, w, 2.0 ** -24, 7)
    assert out.isfinite().all() and ((lse[0, 0].double() - l).abs() <= bound).all()
    # A weight x below FP16's smallest step 2^-24 becomes 0 or, above half of it, 2^-24 < 2 x; larger ones are rounded by less.
    assert (out[0, 0].double().abs() <= 2 * (w @ v.abs()) * (1 + 2.0 ** -8)).all()
