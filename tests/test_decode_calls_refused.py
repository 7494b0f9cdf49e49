"""What the calls around a decode step refuse before anything is launched: through the C interface with addresses that nothing reads, and
through the Python bodies with tensors that are no GPU's (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2607_01831_b200 as lynx

OK, NULL, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 4
P = 1 << 20      # an aligned address


def _spec(tokens=4, pairs=64, axes=1, n_pos=10, axis=0, pos=P, table=P):
    return lynx._RotarySpec(pos, table, tokens, axes, n_pos, pairs, 0, (ctypes.c_uint8 * 64)(*([axis] * 64)))


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _norm_rotary(norm=None, spec=None, width=128, q=P, qs=1024, hq=8, k=P, ks=256, hk=2, T=0, qo=P, qos=1024, ko=P, kos=256):
    return lynx.load().lynx_norm_rotary(_ref(norm), _ref(spec), width, q, qs, hq, k, ks, hk, T, qo, qos, ko, kos, None)


def test_norm_rotary():
    w = lynx._HeadNorm
    assert _norm_rotary() == OK and _norm_rotary(T=4, hq=0, hk=0) == OK
    assert _norm_rotary(T=-1) == SHAPE and _norm_rotary(hq=-1) == SHAPE and _norm_rotary(hq=65536) == SHAPE
    assert _norm_rotary(width=96) == UNSUPPORTED and _norm_rotary(width=512) == UNSUPPORTED
    for bad, want in ((dict(q=None), NULL), (dict(ko=None), NULL), (dict(qs=1023), SHAPE), (dict(qs=1016), SHAPE), (dict(kos=255), SHAPE), (dict(q=P + 8), ALIGN),
                      (dict(ko=P + 2), ALIGN), (dict(width=256), SHAPE), (dict(spec=_spec(3)), SHAPE), (dict(spec=_spec(axes=0)), SHAPE),
                      (dict(spec=_spec(axes=9)), SHAPE), (dict(spec=_spec(n_pos=0)), SHAPE), (dict(spec=_spec(pairs=12)), UNSUPPORTED),
                      (dict(spec=_spec(pairs=72)), UNSUPPORTED), (dict(spec=_spec(axis=1)), SHAPE), (dict(spec=_spec(pos=None)), NULL),
                      (dict(spec=_spec(table=None)), NULL), (dict(spec=_spec(table=P + 4)), ALIGN), (dict(spec=_spec(pos=P + 2)), ALIGN),
                      (dict(width=64, spec=_spec(pairs=40)), SHAPE), (dict(norm=w(P + 8, P, 0.0, 0)), ALIGN), (dict(norm=w(P, P + 4, 0.0, 0)), ALIGN),
                      (dict(norm=w(P, P, -1.0, 0)), SHAPE), (dict(norm=w(None, P, float("nan"), 0)), SHAPE)):
        assert _norm_rotary(**{"T": 4, **bad}) == want, bad


def _shape(**kw):
    return lynx.Geometry(**{**dict(num_q_heads=8, num_kv_heads=2, block_tokens=16, num_blocks=4, max_blocks_per_seq=4), **kw})._c()


def _append(shape=None, k=P, n_src=4, rows=None, n=4, slots=P, norm=None, spec=None, K=(P, P, P), v=P):
    plane = lynx._Plane(*K)
    return lynx.load().lynx_norm_cache_append(_ref(shape or _shape()), k, 256, v, 256, n_src, rows, n, slots, _ref(norm), _ref(spec), plane, plane, None)


def test_norm_cache_append():
    w = lynx._HeadNorm
    assert _append(n=0) == OK and _append(n_src=0, rows=P) == OK
    for bad, want in ((dict(n=-1), SHAPE), (dict(n=5), SHAPE), (dict(shape=_shape(head_dim=64)), UNSUPPORTED), (dict(k=None), NULL), (dict(slots=P + 4), ALIGN),
                      (dict(norm=w(None, P + 8, 0.0, 0)), ALIGN), (dict(norm=w(None, P, -1e-9, 0)), SHAPE), (dict(spec=_spec(3)), SHAPE),
                      (dict(K=(P, None, P)), NULL), (dict(K=(P, P, P + 4)), ALIGN)):
        assert _append(**bad) == want, bad


def _plan(shape=None, old=P, new=P, batch=4, table=P, ring=P, state=P, rows=0, lens=2 * P, offsets=P, slots=P, positions=P):
    return lynx.load().lynx_plan_blocks(_ref(shape or _shape()), old, new, batch, table, ring, state, rows, lens, offsets, slots, positions, None)


def test_plan_blocks():
    for bad, want in ((dict(batch=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(shape=_shape(block_tokens=0)), SHAPE), (dict(shape=_shape(num_blocks=0)), SHAPE),
                      (dict(shape=_shape(max_blocks_per_seq=0)), SHAPE), (dict(old=None), NULL), (dict(new=None), NULL), (dict(table=None), NULL),
                      (dict(lens=None), NULL), (dict(ring=None), NULL), (dict(state=None), NULL), (dict(slots=P + 4), ALIGN), (dict(positions=P + 2), ALIGN),
                      (dict(ring=P + 1), ALIGN), (dict(lens=P), SHAPE), (dict(rows=1 << 31), UNSUPPORTED),
                      (dict(shape=_shape(block_tokens=65536, max_blocks_per_seq=32768)), UNSUPPORTED),
                      (dict(batch=20000, shape=_shape(max_blocks_per_seq=8192)), UNSUPPORTED)):
        assert _plan(**bad) == want, bad
    assert _plan(batch=0, old=None, new=None, table=None, lens=None, offsets=None) == OK      # nothing to do


def _latent(shape=None, c=P, cs=576, k=P, ks=576, n_src=4, rows=None, n=4, slots=P, weight=None, eps=0.0, spec=None, C=(P, P, P), pages=P):
    return lynx.load().lynx_latent_append(_ref(shape or _shape(num_kv_heads=4)), c, cs, k, ks, n_src, rows, n, slots, weight, 0, eps, _ref(spec),
                                          lynx._Plane(*C), pages, None)


def test_latent_rows():
    assert _latent(n=0) == OK and _latent(n_src=0, rows=P) == OK
    for bad, want in ((dict(shape=_shape()), UNSUPPORTED), (dict(shape=_shape(num_kv_heads=4, head_dim=64)), UNSUPPORTED), (dict(n=-1), SHAPE), (dict(n=5), SHAPE),
                      (dict(c=None), NULL), (dict(k=None), NULL), (dict(pages=None), NULL), (dict(C=(P, None, P)), NULL), (dict(cs=504), SHAPE), (dict(ks=60), SHAPE),
                      (dict(cs=580), SHAPE), (dict(c=P + 8), ALIGN), (dict(pages=P + 8), ALIGN), (dict(weight=P + 4), ALIGN), (dict(weight=P, eps=-1.0), SHAPE),
                      (dict(spec=_spec(pairs=64)), SHAPE), (dict(spec=_spec(3, 32)), SHAPE), (dict(slots=P + 4), ALIGN)):
        assert _latent(**bad) == want, bad
    L, plane = lynx.load(), lynx._Plane(P, None, P)
    s = _shape(num_kv_heads=4)
    read = lambda shape=s, C=plane, pages=P, table=P, B=1, starts=None, offsets=P, n=4, out=P, keys=P: L.lynx_latent_read(
        _ref(shape), C, pages, table, B, starts, offsets, n, out, keys, None)
    assert read(n=0) == OK
    for bad, want in ((dict(n=-1), SHAPE), (dict(B=0), SHAPE), (dict(shape=_shape()), UNSUPPORTED), (dict(shape=_shape(num_kv_heads=4, max_blocks_per_seq=0)), SHAPE),
                      (dict(C=lynx._Plane(None, None, P)), NULL), (dict(pages=None), NULL), (dict(offsets=None), NULL), (dict(out=None), NULL), (dict(keys=None), NULL),
                      (dict(out=P + 8), ALIGN), (dict(pages=P + 8), ALIGN), (dict(offsets=P + 1), ALIGN)):
        assert read(**bad) == want, bad


def _attend(shape=None, q=P, qs=576, qr=P, qrs=576, B=2, n=1, C=(P, P, P), pages=P, table=P, lens=P, scale=0.0, out=P, lse=None, ws=P, nbytes=1 << 30):
    return lynx.load().lynx_latent_attention(_ref(shape or _shape(num_kv_heads=4)), q, qs, qr, qrs, B, n, 1, lynx._Plane(*C), pages, table, lens, scale, 0, out, lse, ws,
                                             nbytes, None)


def test_latent_attention():
    lat = lambda **kw: _shape(**{"num_kv_heads": 4, **kw})
    assert _attend(B=0) == OK
    for bad, want in ((dict(B=-1), SHAPE), (dict(n=0), SHAPE), (dict(shape=lat(num_q_heads=0)), SHAPE), (dict(shape=lat(max_blocks_per_seq=0)), SHAPE),
                      (dict(shape=_shape()), UNSUPPORTED), (dict(shape=lat(head_dim=64)), UNSUPPORTED), (dict(shape=lat(block_tokens=24)), UNSUPPORTED),
                      (dict(shape=lat(num_q_heads=129)), UNSUPPORTED), (dict(n=65), UNSUPPORTED), (dict(shape=lat(num_blocks=1 << 26)), UNSUPPORTED),
                      (dict(shape=lat(max_blocks_per_seq=1 << 26)), UNSUPPORTED), (dict(B=1 << 22), UNSUPPORTED),
                      (dict(q=None), NULL), (dict(qr=None), NULL), (dict(C=(None, P, P)), NULL), (dict(C=(P, P, None)), NULL), (dict(pages=None), NULL),
                      (dict(table=None), NULL), (dict(lens=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(qs=504), SHAPE), (dict(qrs=56), SHAPE),
                      (dict(qs=578), SHAPE), (dict(q=P + 8), ALIGN), (dict(qr=P + 2), ALIGN), (dict(C=(P, P + 8, P)), ALIGN), (dict(C=(P, P, P + 4)), ALIGN),
                      (dict(pages=P + 8), ALIGN), (dict(out=P + 8), ALIGN), (dict(lse=P + 2), ALIGN), (dict(table=P + 1), ALIGN), (dict(lens=P + 2), ALIGN),
                      (dict(ws=P + 8), ALIGN)):
        assert _attend(**bad) == want, bad
    need = lynx.load().lynx_latent_workspace_bytes(ctypes.byref(lat()), 2, 1)
    assert need > 0 and _attend(nbytes=need - 1) == 5      # (LYNX_ERR_WORKSPACE)


def test_a_latent_workspace_serves_smaller_calls():
    size = lambda B, n, **kw: lynx.latent_workspace_bytes(lynx.Geometry(**{**dict(num_q_heads=16, num_kv_heads=4, block_tokens=16, num_blocks=99, max_blocks_per_seq=40), **kw}),
                                                          B, n)
    for kw in ({}, dict(max_blocks_per_seq=8), dict(num_q_heads=128), dict(num_q_heads=1), dict(max_blocks_per_seq=4000)):
        for B in (1, 2, 3, 5, 31, 147, 148, 149, 700):
            for n in (1, 2, 3, 4, 5, 8, 9, 63, 64):
                here = size(B, n, **kw)
                assert here > 0 and size(B + 1, n, **kw) >= here
                if n < 64:
                    assert size(B, n + 1, **kw) >= here
    assert size(1, 65) == 0 and size(0, 1) == 0 and size(1, 1, num_kv_heads=2) == 0
    with pytest.raises(lynx.LynxError, match="unsupported"):
        lynx.make_latent_workspace(lynx.Geometry(16, 2, 16, 4, 4), 1, 1, "cpu")


def test_the_python_bodies():
    E = lynx.LynxError
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    geo, lat = lynx.Geometry(8, 2, 16, 4, 4), lynx.Geometry(16, 4, 16, 4, 4)
    planes, latents, pages = lynx.alloc_planes((4, 2, 16), "cpu"), lynx.alloc_planes((4, 4, 16), "cpu"), bf(4, 16, 64)
    k, slots, pool = bf(3, 2, 128), torch.zeros(3, dtype=torch.int64), lynx.make_block_pool(4, "cpu")
    assert pool.ring.tolist() == [0, 1, 2, 3] and pool.state.tolist() == [0, 4, 0, 0]
    for weights in ((bf(128), torch.zeros(128)), (bf(128), bf(64)), (bf(2, 64), None), (None, i32(128))):
        with pytest.raises(E, match="weights"):
            lynx.HeadNorm(*weights)
    with pytest.raises(E, match="eps"):
        lynx.HeadNorm(bf(128), eps=-1.0)
    norm = lynx.HeadNorm(bf(128), bf(128), 1)
    assert norm.eps == 1.0

    def attend(geo=lat, q=bf(1, 1, 16, 512), qr=bf(1, 1, 16, 64), C=latents, pages=pages, table=i32(1, 4), lens=i32(1), **kw):
        return lynx.latent_attention(geo, q, qr, C, pages, table, lens, torch.zeros(1 << 16, dtype=torch.uint8), **kw)

    calls = [
        ("device", lambda: lynx.norm_rotary(k, k, norm)),
        ("needed", lambda: lynx.norm_rotary(None, None, norm)),
        ("64, 128 or 256", lambda: lynx.norm_rotary(bf(3, 2, 96), None)),
        ("as many tokens", lambda: lynx.norm_rotary(None, k, norm, k_out=k[:2])),
        ("BF16", lambda: lynx.norm_rotary(k.float(), None, norm)),
        ("128 values", lambda: lynx.HeadNorm(bf(64))._c(128)),
        ("device", lambda: lynx.cache_append(geo, k, k, slots, planes, planes, norm=norm)),
        ("device", lambda: lynx.plan_blocks(geo, pool, i32(2, 4), i32(2), i32(2), 8)),
        ("block_table", lambda: lynx.plan_blocks(geo, pool, i32(2, 3), i32(2), i32(2), 8)),
        ("old_lens", lambda: lynx.plan_blocks(geo, pool, i32(2, 4), i32(3), i32(2), 8)),
        ("old_lens", lambda: lynx.plan_blocks(geo, pool, i32(2, 4), i32(2), i32(2).long(), 8)),
        ("pool", lambda: lynx.plan_blocks(geo, lynx.make_block_pool(5, "cpu"), i32(2, 4), i32(2), i32(2), 8)),
        ("max_tokens", lambda: lynx.plan_blocks(geo, pool, i32(2, 4), i32(2), i32(2), -1)),
        ("device", lambda: lynx.latent_append(lat, bf(3, 512), bf(3, 64), slots, latents, pages)),
        ("latents", lambda: lynx.latent_append(lat, bf(3, 500), bf(3, 64), slots, latents, pages)),
        ("device|rope_keys", lambda: lynx.latent_append(lat, bf(3, 512), bf(3, 32), slots, latents, pages)),
        ("device", lambda: lynx.latent_read(lat, latents, pages, i32(1, 4), None, i32(2), 3)),
        ("offsets", lambda: lynx.latent_read(lat, latents, pages, i32(1, 4), None, i32(3), 3)),
        ("num_kv_heads", lambda: lynx.latent_read(geo, planes, pages, i32(1, 4), None, i32(2), 3)),
        ("rope_pages", lambda: lynx.latent_read(lat, latents, pages[:3], i32(1, 4), None, i32(2), 3)),
        ("Residual", lambda: lynx.latent_read(lat, lynx.Planes(latents.anchor, None, latents.meta), pages, i32(1, 4), None, i32(2), 3)),
        ("n_rows", lambda: lynx.latent_read(lat, latents, pages, i32(1, 4), None, i32(2), -1)),
        ("device", lambda: attend()),
        ("q_latent", lambda: attend(q=bf(1, 1, 15, 512))),
        ("q_latent", lambda: attend(q=torch.zeros(1, 1, 16, 512))),
        ("device|q_rope", lambda: attend(qr=bf(1, 1, 16, 32))),
        ("block_table", lambda: attend(table=i32(1, 5))),
        ("seq_lens", lambda: attend(lens=i32(2))),
        ("out", lambda: attend(out=torch.zeros(1, 1, 16, 512, dtype=torch.float16))),
        ("lse", lambda: attend(lse=torch.zeros(1, 16))),
        ("Residual", lambda: attend(C=lynx.Planes(latents.anchor, None, latents.meta))),
        ("num_kv_heads", lambda: attend(geo=lynx.Geometry(16, 2, 16, 4, 4))),
        ("rope_pages", lambda: attend(pages=pages[:3])),
    ]
    for match, call in calls:
        with pytest.raises(E, match=match):
            call()
