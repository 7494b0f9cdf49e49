"""Norms of heads with rotary positions, alone and on the way into the cache, against 64 bits.

Bounds.  A head's sum of squares is a chain of 8 FP32 fused additions and at most 5 more, all terms positive: 13 roundings, 13 * 2^-24 of it; mean + eps
one more, half of that in the square root, rsqrtf 2 units of the last place (2^-22): 2^-20.4 of the factor.  Two products (2^-23), and the turn's three
roundings (2^-22) of its terms: below 2^-19 of |y1 c| + |y2 s|, 2^-18 with the BF16 step's share of it.  One rounding to BF16, 2^-8 of the value.
Appended keys are those FP32 values, quantised: the planes' zero + scale * code is within scale / 2 of them, and what FP32 does to scale, zero, the
reciprocal and the difference is below 2^-20 of the row's largest: 2^-17 of it covers both."""
import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf16(*shape, seed=0, spread=1.0):
    return (torch.randn(*shape, generator=_gen(seed)) * spread).to(torch.bfloat16)


def _spec(tokens, pairs, axes=1, interleaved=False, mixed=False, seed=0, n_pos=700):
    pos = torch.randint(0, n_pos, (axes, tokens), generator=_gen(seed), dtype=torch.int32)
    table = lynx.rotary_table(n_pos, pairs, 10000.0)
    axis = [(i if mixed else i * axes // pairs) % axes for i in range(pairs)]
    return lynx.Rotary(pos.cuda(), table.cuda(), axis, interleaved), (pos, table, axis, interleaved)


def _norm64(x, w, eps=EPS):
    if w is None:
        return x
    eps = float(torch.tensor(eps, dtype=torch.float32))
    return x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()


def _turn64(x, host):
    """(turned rows, |y1 c| + |y2 s| at most) of float64 [T][H][W]."""
    if host is None:
        return x, x.abs()
    pos, table, axis, inter = host
    pairs = len(axis)
    p = pos.clamp(0, table.shape[0] - 1).long()
    at = torch.stack([p[a] for a in axis], 1)
    c, s = (table[:, o:o + pairs].double().gather(0, at)[:, None] for o in (0, pairs))
    i1 = torch.arange(pairs) * 2 if inter else torch.arange(pairs)
    i2 = i1 + 1 if inter else i1 + pairs
    y, big = x.clone(), x.abs().clone()
    y[..., i1] = x[..., i1] * c - x[..., i2] * s
    y[..., i2] = x[..., i2] * c + x[..., i1] * s
    big[..., i1] = big[..., i2] = x[..., i1].abs() + x[..., i2].abs()
    return y, big


def _close(got, x, w, host, eps=EPS):
    want, big = _turn64(_norm64(x.double(), w, eps), host)
    assert ((got.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * big).all()


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 1), (3, 32, 8), (5, 7, 1), (130, 64, 8), (2501, 12, 3)])
@pytest.mark.parametrize("W,pairs,axes,inter,mixed", [(128, 64, 1, False, False), (128, 64, 3, True, True), (128, 16, 2, False, True), (64, 32, 1, False, False),
                                                      (64, 8, 1, True, False), (64, 32, 3, True, True), (256, 64, 3, False, False), (256, 64, 1, True, False)])
@pytest.mark.parametrize("floats", [False, True])
def test_norm_and_positions(T, Hq, Hkv, W, pairs, axes, inter, mixed, floats):
    spec, host = _spec(T, pairs, axes, inter, mixed, seed=T + pairs)
    wq, wk = ((1 + 0.3 * torch.randn(W, generator=_gen(i + W))).to(torch.float32 if floats else torch.bfloat16) for i in range(2))
    norm = lynx.HeadNorm(wq.cuda(), wk.cuda(), EPS)
    qkv = _bf16(T, Hq + 2 * Hkv, W, seed=T)
    qkv[0, 0], qkv[-1, Hq] = 0.0, 3.0e4        # a row of zeros, one of large equal values
    d = qkv.cuda()
    before = d.clone()
    q, k = lynx.norm_rotary(d[:, :Hq], d[:, Hq:Hq + Hkv], norm, spec)
    assert torch.equal(d, before) and q.is_contiguous() and k.is_contiguous()
    _close(q, qkv[:, :Hq], wq, host)
    _close(k, qkv[:, Hq:Hq + Hkv], wk, host)
    # in place, in the fused buffer; the values stay
    lynx.norm_rotary(d[:, :Hq], d[:, Hq:Hq + Hkv], norm, spec, q_out=d[:, :Hq], k_out=d[:, Hq:Hq + Hkv])
    assert torch.equal(d[:, :Hq], q) and torch.equal(d[:, Hq:Hq + Hkv], k) and torch.equal(d[:, Hq + Hkv:], before[:, Hq + Hkv:])


@pytest.mark.parametrize("W", [64, 128, 256])
def test_either_part_alone(W):
    T, H = 77, 5
    x = _bf16(T, H, W, seed=W)
    w = _bf16(W, seed=1)
    spec, host = _spec(T, W // 4, 1, seed=2)
    d = x.cuda()
    _close(lynx.norm_rotary(d, None, lynx.HeadNorm(w.cuda()))[0], x, w, None)
    q, k = lynx.norm_rotary(d, d, lynx.HeadNorm(None, w.cuda()), spec)           # keys normed alone
    _close(q, x, None, host)
    _close(k, x, w, host)
    assert torch.equal(lynx.norm_rotary(None, d)[1], d)                          # a copy
    assert torch.equal(lynx.norm_rotary(d, None, None, spec)[0], q)
    if W == 128:
        assert torch.equal(lynx.rotary(d, None, spec)[0], q)
    a, b = lynx.norm_rotary(d[:0], d[:0], lynx.HeadNorm(w.cuda(), w.cuda()), spec)
    assert a.shape == b.shape == (0, H, W)


def test_rows_are_apart():
    """A row that is no number spoils itself alone; tiny and huge rows keep their digits."""
    T, H, W = 13, 6, 128
    x = _bf16(T, H, W, seed=4)
    x[1] *= 2.0 ** -60
    x[2] *= 2.0 ** 50
    w = _bf16(W, seed=5)
    norm = lynx.HeadNorm(w.cuda(), None, 0.0)
    q, _ = lynx.norm_rotary(x.cuda(), None, norm)
    _close(q, x, w, None, 0.0)
    x[7, 3, 50], x[8, 2, 0] = float("nan"), float("inf")
    q2, _ = lynx.norm_rotary(x.cuda(), None, norm)
    bad = torch.zeros(T, H, dtype=torch.bool)
    bad[7, 3] = bad[8, 2] = True
    assert torch.equal(q2.cpu()[~bad], q.cpu()[~bad]) and q2.cpu()[7, 3].isnan().all()


def _pool(nb, H, bt, fill=0):
    return lynx.Planes(torch.full((nb, H, bt, 64), fill, dtype=torch.uint8, device="cuda"),
                       torch.full((nb, H, bt, 64), fill, dtype=torch.uint8, device="cuda"),
                       torch.full((nb, H, bt, 2), float(fill), device="cuda"))


def _same(a, b):
    return all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("anchor", "residual", "meta"))


@pytest.mark.parametrize("T,H,bt", [(1, 1, 16), (7, 8, 5), (61, 3, 64), (5000, 8, 16)])
@pytest.mark.parametrize("pairs", [0, 64, 24])
@pytest.mark.parametrize("picked", [False, True])
def test_normed_keys_into_the_cache(T, H, bt, pairs, picked):
    nb = (T + bt - 1) // bt + 3
    slots = torch.randperm(nb * bt, generator=_gen(T))[:T]
    given = slots.clone()
    given[torch.rand(T, generator=_gen(T + 1)) < 0.1] = -1
    rows = torch.randint(0, T, (T,), generator=_gen(3), dtype=torch.int32) if picked else None
    spec, host = _spec(T, pairs, 1, pairs == 24, seed=T) if pairs else (None, None)
    x = _bf16(T, 2 * H, 128, seed=T + 2, spread=3.0)
    d, w = x.cuda(), _bf16(128, seed=9)
    geo = lynx.Geometry(H, H, bt, nb, 1)
    K, V, K2, V2 = (_pool(nb, H, bt) for _ in range(4))
    r = None if rows is None else rows.cuda()
    lynx.cache_append(geo, d[:, :H], d[:, H:], given.cuda(), K, V, rows=r, rotary=spec, norm=lynx.HeadNorm(None, w.cuda(), EPS))
    lynx.cache_append(geo, d[:, :H], d[:, H:], given.cuda(), K2, V2, rows=r, rotary=spec)
    assert _same(V, V2)
    K3, V3 = _pool(nb, H, bt), _pool(nb, H, bt)
    lynx.cache_append(geo, d[:, :H], d[:, H:], given.cuda(), K3, V3, rows=r, rotary=spec, norm=lynx.HeadNorm(w.cuda(), None))
    assert _same(K3, K2) and _same(V3, V2)
    y = _turn64(_norm64(x[:, :H].double(), w), host)[0]
    y = y if rows is None else y[rows.long()]
    live = given >= 0
    at = given[live]
    code = lynx.recombine(K)[0].cpu()[at // bt, :, at % bt].double()
    meta = K.meta.cpu()[at // bt, :, at % bt].double()
    big = y[live].abs().amax(-1, keepdim=True)
    assert ((meta[..., 1:] + meta[..., :1] * code - y[live]).abs() <= meta[..., :1] / 2 + 2.0 ** -17 * big).all()
    span = y[live].amax(-1, keepdim=True) - y[live].amin(-1, keepdim=True)
    assert ((meta[..., :1] * 255 - span).abs() <= 2.0 ** -17 * big).all()
    untouched = torch.ones(nb * bt, dtype=torch.bool)
    untouched[at] = False
    for t in (K.anchor, K.residual, K.meta):
        assert (t.cpu().transpose(1, 2).flatten(0, 1)[untouched] == 0).all()


def test_the_extension_and_the_python_bodies_agree(monkeypatch):
    T, H, bt, nb = 37, 4, 16, 8
    spec, _ = _spec(T, 64, 3, seed=5)
    d = _bf16(T, 8 * H, 128, seed=6).cuda()
    norm = lynx.HeadNorm(_bf16(128, seed=7).cuda(), _bf16(128, seed=8).cuda())
    slots = torch.randperm(nb * bt, generator=_gen(1))[:T].cuda()
    geo = lynx.Geometry(H, H, bt, nb, nb)

    def calls():
        K, V = _pool(nb, H, bt), _pool(nb, H, bt)
        q, k = lynx.norm_rotary(d[:, :6 * H], d[:, 6 * H:7 * H], norm, spec)
        own = torch.empty_like(k)
        assert lynx.norm_rotary(None, d[:, 6 * H:7 * H], norm, None, k_out=own)[1] is own
        lynx.cache_append(geo, d[:, 6 * H:7 * H], d[:, 7 * H:], slots, K, V, rotary=spec, norm=norm)
        return [q, k, own, K.anchor, K.residual, K.meta, V.anchor]
    fast = calls()
    for name in ("_fast_norm_rotary", "_fast_norm_append"):
        monkeypatch.setattr(lynx, name, lynx._python_only)
    assert all(torch.equal(a, b) for a, b in zip(fast, calls()))
