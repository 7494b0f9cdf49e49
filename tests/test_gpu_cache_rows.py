"""Rotary positions, tokens written into the planes and read back, against 64 bits and the CPU oracle.

Bounds.  Rotary: one rounding to BF16 (2^-8 of the result at most) behind FP32 products and a sum (3 roundings of 2^-24 of the
terms; 2^-22 covers them).  Unrotated appends are the oracle's planes bit for bit, reads its BF16 rows bit for bit.  Rotated keys are FP32
values a few 2^-24 of the row's largest entry off, so that scalars agree to 2^-20 of it and a code differs by one at most, where the
exact quotient lies within 255 * 2^-20 * (largest / range) of a tie."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_01831_b200 as lynx
from util import bf16_bits, dequant

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf16(*shape, seed=0, spread=1.0):
    return (torch.randn(*shape, generator=_gen(seed)) * spread).to(torch.bfloat16)


def _spec(tokens, pairs=64, axes=1, interleaved=False, mixed=False, seed=0, n_pos=700):
    pos = torch.randint(0, n_pos, (axes, tokens), generator=_gen(seed), dtype=torch.int32)
    table = lynx.rotary_table(n_pos, pairs, 10000.0)
    axis = [(i if mixed else i * axes // pairs) % axes for i in range(pairs)]
    return lynx.Rotary(pos.cuda(), table.cuda(), axis, interleaved), (pos, table, axis, interleaved)


def _turn64(x, host):
    """x float64 [T][H][128]; the pairs of channels as complex numbers."""
    pos, table, axis, inter = host
    pairs = len(axis)
    p = pos.clamp(0, table.shape[0] - 1).long()
    at = torch.stack([p[a] for a in axis], 1)
    c, s = (table[:, o:o + pairs].double().gather(0, at)[:, None] for o in (0, pairs))
    y = x.clone()
    i1 = torch.arange(pairs) * 2 if inter else torch.arange(pairs)
    i2 = i1 + 1 if inter else i1 + pairs
    y[..., i1] = x[..., i1] * c - x[..., i2] * s
    y[..., i2] = x[..., i2] * c + x[..., i1] * s
    big = x.abs().clone()
    big[..., i1] = big[..., i2] = x[..., i1].abs() + x[..., i2].abs()
    return y, big


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 1), (3, 32, 8), (5, 7, 1), (130, 64, 8), (3001, 12, 3)])
@pytest.mark.parametrize("pairs,axes,inter,mixed", [(64, 1, False, False), (64, 3, False, False), (64, 3, True, True), (16, 2, False, True),
                                                    (8, 1, True, False), (40, 1, False, False)])
def test_rotary(T, Hq, Hkv, pairs, axes, inter, mixed):
    spec, host = _spec(T, pairs, axes, inter, mixed, seed=T + pairs)
    qkv = _bf16(T, Hq + 2 * Hkv, 128, seed=T)
    d = qkv.cuda()
    before = d.clone()
    q, k = lynx.rotary(d[:, :Hq], d[:, Hq:Hq + Hkv], spec)
    assert torch.equal(d, before) and q.is_contiguous() and k.is_contiguous()
    for got, x in ((q, qkv[:, :Hq]), (k, qkv[:, Hq:Hq + Hkv])):
        want, big = _turn64(x.double(), host)
        assert ((got.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * big).all()
        assert torch.equal(got[..., 2 * pairs:].cpu(), x[..., 2 * pairs:])
    # in place, in the fused buffer; the values stay out of it
    lynx.rotary(d[:, :Hq], d[:, Hq:Hq + Hkv], spec, q_out=d[:, :Hq], k_out=d[:, Hq:Hq + Hkv])
    assert torch.equal(d[:, :Hq], q) and torch.equal(d[:, Hq:Hq + Hkv], k) and torch.equal(d[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_rotary_one_tensor_and_positions_out_of_range():
    T = 9
    spec, host = _spec(T, n_pos=50)
    x = _bf16(T, 5, 128, seed=3)
    spec.positions[0, 0], spec.positions[0, 1], spec.positions[0, 2] = -7, 50, 2 ** 31 - 1
    want, big = _turn64(x.double(), (spec.positions.cpu(), *host[1:]))
    q, none = lynx.rotary(x.cuda(), None, spec)
    none2, k = lynx.rotary(None, x.cuda(), spec)
    assert none is None and none2 is None and torch.equal(q, k)
    assert ((q.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * big).all()
    q0, k0 = lynx.rotary(x[:0].cuda(), x[:0].cuda(), spec)
    assert q0.shape == (0, 5, 128) and k0.shape == (0, 5, 128)


def _pool(nb, H, bt, fill):
    return lynx.Planes(torch.full((nb, H, bt, 64), fill, dtype=torch.uint8, device="cuda"),
                       torch.full((nb, H, bt, 64), fill, dtype=torch.uint8, device="cuda"),
                       torch.full((nb, H, bt, 2), float(fill), device="cuda"))


def _rows_of(p, slots, bt):
    return [t[slots // bt, :, slots % bt].cpu() for t in (p.anchor, p.residual, p.meta)]


@pytest.mark.parametrize("bt", [1, 5, 16, 64])
@pytest.mark.parametrize("T,H,strided", [(1, 1, False), (7, 8, True), (61, 3, True), (1030, 8, False)])
def test_append_is_the_quantiser(T, H, bt, strided):
    nb = (T + bt - 1) // bt + 3
    slots = torch.randperm(nb * bt, generator=_gen(T))[:T]
    skip = torch.rand(T, generator=_gen(T + 1)) < 0.1
    given = slots.clone()
    given[skip] = torch.tensor([-1, nb * bt, 2 ** 40])[torch.arange(int(skip.sum())) % 3]
    src = _bf16(T, 3 * H, 128, seed=T + 2, spread=30.0)
    src[0, 0], src[-1, H] = 2.5, -0.0     # constant rows
    d = src.cuda()
    k, v = (d[:, :H], d[:, H:2 * H]) if strided else (d[:, :H].contiguous(), d[:, H:2 * H].contiguous())
    K, V = _pool(nb, H, bt, 3), _pool(nb, H, bt, 5)
    lynx.cache_append(lynx.Geometry(H, H, bt, nb, 1), k, v, given.cuda(), K, V)
    for p, x, fill in ((K, src[:, :H], 3), (V, src[:, H:2 * H], 5)):
        want = oracle.split_quantize(bf16_bits(x))
        got = _rows_of(p, slots.cuda(), bt)
        for g, w in zip(got, want):
            w = torch.from_numpy(np.ascontiguousarray(w)).view(g.shape)
            assert torch.equal(g[~skip], w[~skip].to(g.dtype))
        # nothing else was written
        other = torch.ones(nb * bt, dtype=torch.bool)
        other[slots[~skip]] = False
        rest = _rows_of(p, torch.arange(nb * bt)[other].cuda(), bt)
        assert all((t == fill).all() for t in rest)


@pytest.mark.parametrize("inter,axes,mixed,pairs", [(False, 1, False, 64), (True, 3, False, 64), (False, 3, True, 24)])
@pytest.mark.parametrize("T,n,H", [(1, 1, 8), (40, 13, 8), (9, 9, 2), (3000, 3000, 4)])
def test_append_rotated_rows(T, n, H, inter, axes, mixed, pairs):
    bt, nb = 16, n // 16 + 2
    spec, host = _spec(T, pairs, axes, inter, mixed, seed=n)
    k, v = _bf16(T, H, 128, seed=n), _bf16(T, H, 128, seed=n + 1)
    pick = torch.randperm(T, generator=_gen(n))[:n].to(torch.int32)
    slots = torch.randperm(nb * bt, generator=_gen(n + 2))[:n]
    rows = pick.clone()
    if n > 4:
        rows[1], rows[3] = -1, T          # left out
    kept = (rows >= 0) & (rows < T)
    K, V = _pool(nb, H, bt, 0), _pool(nb, H, bt, 0)
    lynx.cache_append(lynx.Geometry(H, H, bt, nb, 1), k.cuda(), v.cuda(), slots.cuda(), K, V, rows=rows.cuda(), rotary=spec)
    want = oracle.split_quantize(bf16_bits(v[pick.long()]))
    got = _rows_of(V, slots.cuda(), bt)
    assert all(torch.equal(g[kept], torch.from_numpy(np.ascontiguousarray(w)).view(g.shape)[kept].to(g.dtype)) for g, w in zip(got, want))
    a, r, m = (t[kept].numpy() for t in _rows_of(K, slots.cuda(), bt))
    y = _turn64(k.double(), host)[0][pick.long()][kept].numpy()
    lo, top = y.min(-1, keepdims=True), np.abs(y).max(-1, keepdims=True)
    span = y.max(-1, keepdims=True) - lo
    eps = 2.0 ** -20 * top
    assert (np.abs(m[..., 1:] - lo) <= eps).all() and (np.abs(m[..., :1] * 255.0 - span) <= 2 * eps).all()
    code = np.stack((a & 15, a >> 4), -1).reshape(y.shape) * 16.0 + np.stack((r & 15, r >> 4), -1).reshape(y.shape)
    exact = (y - lo) / span * 255.0
    slack = 255.0 * 4 * eps / span
    assert (np.abs(code - exact) <= 0.5 + slack).all()
    for p in (K, V):                      # what was left out is untouched
        assert all((t[~kept] == 0).all() for t in _rows_of(p, slots.cuda(), bt))


@pytest.mark.parametrize("bt", [1, 5, 16, 32])
@pytest.mark.parametrize("lens", [(1,), (40, 1, 300), tuple([17, 0, 3] * 30), (2500, 700)])
@pytest.mark.parametrize("anchor_only", [False, True])
def test_read(lens, bt, anchor_only):
    H, B = 3, len(lens)
    g = _gen(sum(lens) + bt)
    need = [max(1, -(-n // bt)) for n in lens]
    nb = sum(need) + 2
    ids = torch.randperm(nb, generator=g).to(torch.int32)
    table = torch.zeros(B, max(need) + 1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = ids[sum(need[:b]):sum(need[:b]) + n]
    x = [_bf16(nb, H, bt, 128, seed=i + bt, spread=5.0) for i in range(2)]
    P = [oracle.split_quantize(bf16_bits(t)) for t in x]
    K, V = (lynx.Planes(*(torch.from_numpy(np.ascontiguousarray(w)).view(nb, H, bt, -1).cuda() for w in p)) for p in P)
    starts = torch.tensor([n // 3 for n in lens], dtype=torch.int32)
    counts = torch.tensor(lens, dtype=torch.int32) - starts
    offsets = torch.cat((torch.zeros(1, dtype=torch.int32), counts.cumsum(0).to(torch.int32)))
    n_rows = int(offsets[-1]) + 6         # the last six belong to no sequence
    geo = lynx.Geometry(H, H, bt, nb, table.shape[1])
    if anchor_only:
        K.residual = V.residual = None
    outs = lynx.cache_read(geo, K, V, table.cuda(), starts.cuda(), offsets.cuda(), n_rows, anchor_only=anchor_only)
    at = torch.cat([s + torch.arange(n) for s, n in zip(starts.tolist(), counts.tolist())]).long()
    seq = torch.repeat_interleave(torch.arange(B), counts.long())
    blk = table[seq, at // bt].long()
    for got, p, planes in zip(outs, P, (K, V)):
        assert got.shape == (n_rows, H, 128) and (got[int(offsets[-1]):] == 0).all()
        a, r, m = (t.reshape(nb, H, bt, -1)[blk, :, at % bt] for t in p)
        # one rounding of the exact code * scale + zero to FP32, one to BF16 (both operands are FP32: the 64-bit sum is exact
        # enough that its FP32 rounding is the fused one's but for ties, which the bound of a BF16 step admits)
        want = dequant(a, r, m, not anchor_only)
        bits = torch.from_numpy(want.astype(np.float32)).to(torch.bfloat16)
        off = got[:int(offsets[-1])].cpu() != bits
        assert off.double().mean() <= 1e-5
        if not anchor_only:
            assert torch.equal(got[:int(offsets[-1])].cpu(), lynx.recombine(planes, False, True)[1].cpu()[blk, :, at % bt])
        assert (np.abs(got[:int(offsets[-1])].cpu().double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 1e-30).all()


def test_read_out_of_range():
    """Tokens past the table, negative ones and block ids outside the pool give zeros; starts may be absent."""
    H, bt, nb = 2, 16, 4
    K, V = _pool(nb, H, bt, 17), _pool(nb, H, bt, 17)
    table = torch.tensor([[0, 1], [2, 99], [-1, 3]], dtype=torch.int32).cuda()
    geo = lynx.Geometry(H, H, bt, nb, 2)
    starts = torch.tensor([20, 10, -8], dtype=torch.int32).cuda()
    offsets = torch.tensor([0, 20, 40, 70], dtype=torch.int32).cuda()
    k, v = lynx.cache_read(geo, K, V, table, starts, offsets, 70)
    live = torch.zeros(70, dtype=torch.bool)
    live[:12], live[20:26], live[64:70] = True, True, True      # 20..31 | 10..15 | (-8..15 dead) 16..21
    for t in (k, v):
        nonzero = (t != 0).reshape(70, -1).cpu()
        assert nonzero[live].all() and not nonzero[~live].any()
    k0, _ = lynx.cache_read(geo, K, V, table[:1].contiguous(), None, torch.tensor([0, 32], dtype=torch.int32).cuda(), 32)
    assert (k0 != 0).all()
    k0, _ = lynx.cache_read(geo, K, V, table[:1].contiguous(), None, torch.tensor([0, 0], dtype=torch.int32).cuda(), 0)
    assert k0.shape == (0, H, 128)


def test_on_another_stream_and_written_then_read():
    """An append and a read of the same tokens, one behind the other on a side stream."""
    H, bt, nb, T = 8, 16, 40, 500
    x = _bf16(T, 2 * H, 128, seed=8)
    slots = torch.arange(T)
    K, V = _pool(nb, H, bt, 0), _pool(nb, H, bt, 0)
    geo = lynx.Geometry(H, H, bt, nb, nb)
    table, offsets = torch.arange(nb, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([0, T], dtype=torch.int32).cuda()
    d, sl = x.cuda(), slots.cuda()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        lynx.cache_append(geo, d[:, :H], d[:, H:], sl, K, V)
        k, v = lynx.cache_read(geo, K, V, table, None, offsets, T)
    st.synchronize()
    for got, t in ((k, x[:, :H]), (v, x[:, H:])):       # the oracle's codes, back in BF16, bit for bit
        want = oracle.recombine(*oracle.split_quantize(bf16_bits(t)), want_bf16=True)[1]
        assert np.array_equal(bf16_bits(got), np.asarray(want).view(np.uint16).reshape(got.shape))


def test_the_extension_and_the_python_bodies_agree(monkeypatch):
    T, H, bt, nb = 37, 4, 16, 8
    spec, _ = _spec(T, 64, 3, seed=5)
    d = _bf16(T, 8 * H, 128, seed=6).cuda()
    slots = torch.randperm(nb * bt, generator=_gen(1))[:T].cuda()
    rows = torch.randint(0, T, (T,), generator=_gen(2), dtype=torch.int32).cuda()
    geo = lynx.Geometry(H, H, bt, nb, nb)
    table, offsets = torch.arange(nb, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([0, nb * bt], dtype=torch.int32).cuda()

    def calls():
        K, V = _pool(nb, H, bt, 0), _pool(nb, H, bt, 0)
        q, k = lynx.rotary(d[:, :6 * H], d[:, 6 * H:7 * H], spec)
        own = torch.empty_like(k)
        assert lynx.rotary(None, k, spec, k_out=own)[1] is own
        lynx.cache_append(geo, k, d[:, 7 * H:], slots, K, V, rows=rows, rotary=spec)
        lynx.cache_append(geo, k, d[:, 7 * H:], slots, V, K)
        return [q, k, own, K.anchor, K.residual, K.meta, V.anchor, *lynx.cache_read(geo, K, V, table, None, offsets, nb * bt),
                *lynx.cache_read(geo, K, V, table, offsets[:1], offsets, nb * bt, anchor_only=True)]
    fast = calls()
    for name in ("_fast_rotary", "_fast_cache_append", "_fast_cache_read"):
        monkeypatch.setattr(lynx, name, lynx._python_only)
    assert all(torch.equal(a, b) for a, b in zip(fast, calls()))


@pytest.mark.parametrize("tokens,H", [(37, 3), (3000, 8)])
@pytest.mark.parametrize("anchor_only", [False, True])
def test_read_into_outputs_of_less_alignment(tokens, H, anchor_only):
    """16 bytes are enough; what lies in front and behind stays."""
    bt, nb = 16, -(-tokens // 16)
    geo = lynx.Geometry(H, H, bt, nb, nb)
    K, V = _pool(nb, H, bt, 0), _pool(nb, H, bt, 0)
    x = _bf16(tokens, 2 * H, 128, seed=8).cuda()
    lynx.cache_append(geo, x[:, :H], x[:, H:], torch.arange(tokens).cuda(), K, V)
    table, offsets = torch.arange(nb, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([0, tokens], dtype=torch.int32).cuda()
    want = lynx.cache_read(geo, K, V, table, None, offsets, tokens, anchor_only=anchor_only)
    buf = [torch.full((tokens * H * 128 + 16,), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = [b[8:-8].view(tokens, H, 128) for b in buf]
    assert views[0].data_ptr() % 32 == 16
    lynx.cache_read(geo, K, V, table, None, offsets, tokens, anchor_only=anchor_only, k_out=views[0], v_out=views[1])
    for b, view, w in zip(buf, views, want):
        assert torch.equal(view, w) and (b[:8] == 9.0).all() and (b[-8:] == 9.0).all()


def test_refusals():
    T, H, bt, nb = 4, 2, 16, 3
    geo = lynx.Geometry(H, H, bt, nb, 2)
    K, V = _pool(nb, H, bt, 0), _pool(nb, H, bt, 0)
    k = _bf16(T, H, 128).cuda()
    slots = torch.arange(T).cuda()
    spec, _ = _spec(T)
    table, offsets = torch.zeros(1, 2, dtype=torch.int32).cuda(), torch.tensor([0, 4], dtype=torch.int32).cuda()
    E = lynx.LynxError
    bad = [
        lambda: lynx.rotary(k.float(), None, spec),
        lambda: lynx.rotary(k.cpu(), None, spec),
        lambda: lynx.rotary(None, None, spec),
        lambda: lynx.rotary(k[..., :64], None, spec),
        lambda: lynx.rotary(k.transpose(0, 1), None, spec),
        lambda: lynx.rotary(k, k[:2], spec),
        lambda: lynx.rotary(k, None, lynx.Rotary(spec.positions[:, :2], spec.cos_sin)),
        lambda: lynx.rotary(k, None, lynx.Rotary(spec.positions.long(), spec.cos_sin)),
        lambda: lynx.rotary(k, None, lynx.Rotary(spec.positions, spec.cos_sin, [1] * 64)),
        lambda: lynx.rotary(k, None, lynx.Rotary(spec.positions, lynx.rotary_table(8, 12, device="cuda"))),     # 12 pairs
        lambda: lynx.rotary(k, None, lynx.Rotary(spec.positions, spec.cos_sin[:0])),
        lambda: lynx.rotary(torch.zeros(T * H * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(T, H, 128), None, spec),
        lambda: lynx.rotary(torch.zeros(T, H * 128 + 4, dtype=torch.bfloat16, device="cuda")[:, :H * 128].unflatten(1, (H, 128)), None, spec),
        lambda: lynx.cache_append(geo, k, k, slots.int(), K, V),
        lambda: lynx.cache_append(geo, k, k[:3], slots, K, V),
        lambda: lynx.cache_append(geo, k[:3], k[:3], slots, K, V),                    # fewer source rows than slots
        lambda: lynx.cache_append(geo, k, k, slots, K, V, rows=slots),
        lambda: lynx.cache_append(lynx.Geometry(H, H, bt, nb + 1, 2), k, k, slots, K, V),
        lambda: lynx.cache_append(lynx.Geometry(H, H, bt, nb, 2, head_dim=64), k, k, slots, K, V),
        lambda: lynx.cache_append(lynx.Geometry(1, 1, bt, nb, 2), k, k, slots, K, V),
        lambda: lynx.cache_append(geo, k, k, slots, lynx.Planes(K.anchor, None, K.meta), V),
        lambda: lynx.cache_read(geo, K, V, table.long(), None, offsets, 4),
        lambda: lynx.cache_read(geo, K, V, table[:, :1], None, offsets, 4),
        lambda: lynx.cache_read(geo, K, V, table, None, offsets.long(), 4),
        lambda: lynx.cache_read(geo, K, V, table, offsets, offsets, 4),
        lambda: lynx.cache_read(geo, K, lynx.Planes(V.anchor, None, V.meta), table, None, offsets, 4),
        lambda: lynx.cache_read(geo, K, V, table, None, offsets, -1),
        lambda: lynx.cache_read(geo, K, V, table, None, offsets, 4, k_out=torch.empty(4, H, 128, device="cuda")),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((E, RuntimeError)):
            f()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
    assert all((t == 0).all() for p in (K, V) for t in (p.anchor, p.residual, p.meta))
