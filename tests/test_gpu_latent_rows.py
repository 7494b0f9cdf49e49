"""Latents and rotary keys written into the planes and read back.

Without a norm the planes are the quantiser's bit for bit, keys without positions copies.  A norm's factor is a sum of 512 squares: a lane's chain of 64 (or
16 in a chain and 5 exchanges) fused additions of positive terms, 67 roundings at most, half of that in the square root and 2 units of rsqrtf:
(34 + 4) * 2^-24; two products: 2^-18.6 of a value.  The planes' zero + scale * code is within scale / 2 of that, and 2^-17 of the row's largest covers it and
what FP32 does to scale, zero and the quotient (2^-20).  Turned keys: three roundings of the terms (2^-22 of them) and one to BF16."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_01831_b200 as lynx
from util import bf16_bits

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf16(*shape, seed=0, spread=1.0):
    return (torch.randn(*shape, generator=_gen(seed)) * spread).to(torch.bfloat16)


def _cache(nb, bt, fill=0):
    p = lynx.Planes(torch.full((nb, 4, bt, 64), fill, dtype=torch.uint8, device="cuda"), torch.full((nb, 4, bt, 64), fill, dtype=torch.uint8, device="cuda"),
                    torch.full((nb, 4, bt, 2), float(fill), device="cuda"))
    return p, torch.full((nb, bt, 64), float(fill), dtype=torch.bfloat16, device="cuda")


def _at(t, slots, bt):
    return t[slots // bt, :, slots % bt].cpu()


@pytest.mark.parametrize("bt", [1, 5, 16, 64])
@pytest.mark.parametrize("T,strided", [(1, False), (7, True), (61, True), (6001, False)])
def test_append_is_the_quantiser(T, strided, bt):
    nb = (T + bt - 1) // bt + 3
    slots = torch.randperm(nb * bt, generator=_gen(T))[:T]
    skip = torch.rand(T, generator=_gen(T + 1)) < 0.1
    given = slots.clone()
    given[skip] = torch.tensor([-1, nb * bt, 2 ** 40])[torch.arange(int(skip.sum())) % 3]
    src = _bf16(T, 576, seed=T + 2, spread=30.0)
    src[0, :128], src[-1, 128:256] = 2.5, -0.0     # constant rows
    d = src.cuda()
    c, k = (d[:, :512], d[:, 512:]) if strided else (d[:, :512].contiguous(), d[:, 512:].contiguous())
    C, pages = _cache(nb, bt, 3)
    geo = lynx.Geometry(16, 4, bt, nb, 1)
    lynx.latent_append(geo, c, k, given.cuda(), C, pages)
    want = oracle.split_quantize(bf16_bits(src[:, :512].unflatten(1, (4, 128)).contiguous()))
    at = slots.cuda()
    for t, w in zip((C.anchor, C.residual, C.meta), want):
        g, w = _at(t, at, bt), torch.from_numpy(np.ascontiguousarray(w)).view(T, 4, -1)
        assert torch.equal(g[~skip], w[~skip]) and (g[skip] == 3).all()
    got = pages[at // bt, at % bt].cpu()
    assert torch.equal(got[~skip], src[~skip, 512:]) and (got[skip] == 3).all()
    rest = torch.ones(nb * bt, dtype=torch.bool)
    rest[slots] = False
    assert (pages.flatten(0, 1).cpu()[rest] == 3).all() and (C.anchor.cpu().transpose(1, 2).flatten(0, 1)[rest] == 3).all()


@pytest.mark.parametrize("T", [1, 9, 300, 5003])
@pytest.mark.parametrize("pairs,inter,axes", [(32, True, 1), (32, False, 1), (8, False, 2), (24, True, 3), (16, False, 1), (0, False, 1)])
@pytest.mark.parametrize("floats", [False, True])
def test_norm_and_positions(T, pairs, inter, axes, floats):
    bt, eps = 16, 1e-5
    nb = T // bt + 2
    slots = torch.randperm(nb * bt, generator=_gen(T))[:T]
    rows = torch.randint(0, T, (T,), generator=_gen(T + 5), dtype=torch.int32)
    src, w = _bf16(T, 576, seed=T, spread=2.0), (1 + 0.3 * torch.randn(512, generator=_gen(3))).to(torch.float32 if floats else torch.bfloat16)
    d = src.cuda()
    spec = host = None
    if pairs:
        pos, table = torch.randint(0, 300, (axes, T), generator=_gen(T + 1), dtype=torch.int32), lynx.rotary_table(300, pairs, 10000.0)
        axis = [i % axes for i in range(pairs)]
        spec = lynx.Rotary(pos.cuda(), table.cuda(), axis, inter)
    C, pages = _cache(nb, bt)
    lynx.latent_append(lynx.Geometry(16, 4, bt, nb, 1), d[:, :512], d[:, 512:], slots.cuda(), C, pages, weight=w.cuda(), eps=eps, rows=rows.cuda(), rotary=spec)
    x = src[rows.long()].double()
    y = x[:, :512]
    y = (y / (y.square().mean(1, keepdim=True) + float(torch.tensor(eps))).sqrt() * w.double()).unflatten(1, (4, 128))
    code, meta = _at(lynx.recombine(C)[0], slots.cuda(), bt).double(), _at(C.meta, slots.cuda(), bt).double()
    big = y.abs().amax(-1, keepdim=True)
    assert ((meta[..., 1:] + meta[..., :1] * code - y).abs() <= meta[..., :1] / 2 + 2.0 ** -17 * big).all()
    assert ((meta[..., :1] * 255 - (y.amax(-1, keepdim=True) - y.amin(-1, keepdim=True))).abs() <= 2.0 ** -17 * big).all()
    want, most = x[:, 512:].clone(), x[:, 512:].abs()
    if pairs:
        at = torch.stack([pos[a] for a in axis], 1).long()[rows.long()]
        c, s = (table[:, o:o + pairs].double().gather(0, at) for o in (0, pairs))
        i1 = torch.arange(pairs) * 2 if inter else torch.arange(pairs)
        i2 = i1 + 1 if inter else i1 + pairs
        z = x[:, 512:]
        want[:, i1] = z[:, i1] * c - z[:, i2] * s
        want[:, i2] = z[:, i2] * c + z[:, i1] * s
        most[:, i1] = most[:, i2] = z[:, i1].abs() + z[:, i2].abs()
    got = pages.cpu()[slots // bt, slots % bt].double()
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * most).all()


@pytest.mark.parametrize("bt", [1, 5, 16, 32])
@pytest.mark.parametrize("lens", [(1,), (40, 1, 300), tuple([17, 0, 3] * 30), (4900, 700)])
@pytest.mark.parametrize("anchor_only", [False, True])
def test_read(lens, bt, anchor_only):
    B, g = len(lens), _gen(sum(lens) + bt)
    need = [max(1, -(-n // bt)) for n in lens]
    nb = sum(need) + 2
    ids = torch.randperm(nb, generator=g).to(torch.int32)
    table = torch.zeros(B, max(need) + 1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = ids[sum(need[:b]):sum(need[:b]) + n]
    C = lynx.split_quantize(_bf16(nb, 4, bt, 128, seed=bt, spread=5.0).cuda())       # (a pool as the transfer brings it)
    pages = _bf16(nb, bt, 64, seed=bt + 1).cuda()
    starts = torch.tensor([n // 3 for n in lens], dtype=torch.int32)
    counts = torch.tensor(lens, dtype=torch.int32) - starts
    offsets = torch.cat((torch.zeros(1, dtype=torch.int32), counts.cumsum(0).to(torch.int32)))
    n_rows = int(offsets[-1]) + 6         # the last six belong to no sequence
    geo = lynx.Geometry(16, 4, bt, nb, table.shape[1])
    args = table.cuda(), starts.cuda(), offsets.cuda(), n_rows
    c, k = lynx.latent_read(geo, C, pages, *args, anchor_only=anchor_only)
    as_rows = lynx.cache_read(geo, C, C, *args, anchor_only=anchor_only)[0]
    assert torch.equal(c, as_rows.flatten(1))
    at = torch.cat([s + torch.arange(n) for s, n in zip(starts.tolist(), counts.tolist())]).long()
    seq = torch.repeat_interleave(torch.arange(B), counts.long())
    blk = table[seq, at // bt].long()
    assert torch.equal(k[:int(offsets[-1])].cpu(), pages.cpu()[blk, at % bt]) and (k[int(offsets[-1]):] == 0).all()


def test_read_out_of_range():
    bt, nb = 16, 4
    C, pages = _cache(nb, bt, 17)
    table = torch.tensor([[0, 1], [2, 99], [-1, 3]], dtype=torch.int32).cuda()
    starts = torch.tensor([20, 10, -8], dtype=torch.int32).cuda()
    offsets = torch.tensor([0, 20, 40, 70], dtype=torch.int32).cuda()
    live = torch.zeros(70, dtype=torch.bool)
    live[:12], live[20:26], live[64:70] = True, True, True      # 20..31 | 10..15 | (-8..15 dead) 16..21
    for t in lynx.latent_read(lynx.Geometry(16, 4, bt, nb, 2), C, pages, table, starts, offsets, 70):
        assert (t != 0).cpu()[live].all() and not (t != 0).cpu()[~live].any()


def test_the_extension_and_the_python_bodies_agree(monkeypatch):
    T, bt, nb = 37, 16, 4
    d, w = _bf16(T, 576, seed=6).cuda(), _bf16(512, seed=7).cuda()
    spec = lynx.Rotary(torch.arange(T, dtype=torch.int32).cuda(), lynx.rotary_table(T, 32).cuda())
    slots = torch.randperm(nb * bt, generator=_gen(1))[:T].cuda()
    geo = lynx.Geometry(16, 4, bt, nb, nb)
    table, offsets = torch.arange(nb, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([0, nb * bt], dtype=torch.int32).cuda()

    def calls():
        C, pages = _cache(nb, bt)
        st = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            lynx.latent_append(geo, d[:, :512], d[:, 512:], slots, C, pages, weight=w, rotary=spec)
            r = lynx.latent_read(geo, C, pages, table, None, offsets, nb * bt)
        st.synchronize()
        return [C.anchor, C.residual, C.meta, pages, *r]
    fast = calls()
    for name in ("_fast_latent_append", "_fast_latent_read"):
        monkeypatch.setattr(lynx, name, lynx._python_only)
    assert all(torch.equal(a, b) for a, b in zip(fast, calls()))
