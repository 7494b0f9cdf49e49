"""Timed cases of what a decode step does around and on the quantised cache: block tables and slots from request lengths, norms of heads
with their rotary positions, tokens normed on their way into the cache, and caches of latents with the attention that reads them.

A serving step in order: the lengths that the scheduler wants give each request its blocks and each new token its slot; projections are
normed head by head, rotated and quantised into their slots; attention reads the planes.  Models whose keys and values are one
latent vector of 512 channels (four rows of the planes) and one rotary key of 64 a token keep them the same way.  Shapes are those of the
repository's other workloads: 8 KV heads of 128 channels with 32 or 64 query heads, or 16 to 128 query heads on one latent, contexts up to
131072 tokens, blocks of 16 tokens (32 and 64 among the drawn cases), uniform or ragged batches.

`own` false: elementary torch operations in 32 bits.  `own` true: the library's entry points.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
LATENT, ROPE = 512, 64                    # channels of a latent and of its rotary key
SECTIONS = {1: (64,), 3: (16, 24, 24)}    # rotary pairs per axis: positions of text, or time, height and width
EPS = 1e-6


def listed():
    cases = [
        # Norms and rotary positions of one step's tree nodes: 4 sequences x 7 nodes, positions of text.
        dict(name="norm_nodes_28", kind="norm", tokens=28),
        # A long prompt made of images: time, height and width, 64 query heads.
        dict(name="norm_images_32k", kind="norm", tokens=32768, axes=3, group=8, side=48),
        # A decode step of 16 ragged sequences: one token each, keys normed and rotated, quantised into its slot, and read back.
        dict(name="norm_append_decode_16", kind="append", batch=16, new=1, ctx_lo=500, ctx=4000),
        # A prompt of 32768 tokens with image positions into scattered blocks, and read back.
        dict(name="norm_append_prompt_32k", kind="append", batch=1, new=32768, ctx_lo=0, ctx=0, axes=3, side=32),
        # A decode step's windows of 4 drafted tokens for 64 requests get their blocks and slots, and give the blocks back.
        dict(name="plan_windows_64x4", kind="plan", batch=64, new_lo=4, new=4, ctx_lo=500, ctx=8000),
        # Prompts of a large ragged batch (some 130000 tokens) get theirs, and give them back.
        dict(name="plan_prompts_1024", kind="plan", batch=1024, new_lo=1, new=256, ctx_lo=0, ctx=8000),
        # A decode step of 16 sequences of latents: one token each, normed, rotated, quantised into its slot, and read back.
        dict(name="latent_append_decode_16", kind="latent_rows", batch=16, new=1, ctx_lo=500, ctx=4000),
        # A prompt of 32768 tokens of latents into scattered blocks, and read back.
        dict(name="latent_append_prompt_32k", kind="latent_rows", batch=1, new=32768, ctx_lo=0, ctx=0, interleaved=False),
        # One token over a short cache of latents: the smallest call.
        dict(name="latent_16_ctx_300", kind="latent", batch=1, n=1, heads_q=16, ctx_lo=300, ctx=300),
        # Drafting on the Anchor plane alone over one long context, 16 query heads: memory's case.
        dict(name="latent_16_128k_anchor", kind="latent", batch=1, n=1, heads_q=16, ctx_lo=131072, ctx=131072, anchor=True, shuffled=False),
        # A verification window of 4 positions of 8 ragged sequences, 32 query heads.
        dict(name="latent_32x4_mix", kind="latent", batch=8, n=4, heads_q=32, ctx_lo=2000, ctx=32768),
        # A decode step of 128 query heads over a serving mix of 16 ragged sequences: the largest.
        dict(name="latent_128_mix", kind="latent", batch=16, n=1, heads_q=128, ctx_lo=8192, ctx=65536),
    ]
    return [_full(c) for c in cases]


def _full(c):
    """Every option of a case spelt out.  ctx_lo < ctx: ragged lengths, drawn from lens_seed."""
    base = dict(lens_seed=1)
    if c["kind"] in ("norm", "append"):
        base.update(heads=8, group=4, axes=1, side=16, interleaved=False)
    if c["kind"] == "latent_rows":
        base.update(interleaved=True)
    if c["kind"] != "norm":
        base.update(batch=1, block=16, shuffled=True)
    if c["kind"] in ("latent", "latent_rows"):
        base.update(anchor=False)
    return {**base, **c}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    kind = rng.choice(["norm", "append", "plan", "latent_rows", "latent", "latent", "latent"])
    c = dict(kind=kind, lens_seed=rng.randint(1, 1000))
    if kind in ("norm", "append"):
        c.update(group=rng.choice([4, 4, 8, 8, 1, 2]), axes=rng.choice([1, 3]), side=rng.randint(3, 64), interleaved=rng.random() < 0.3)
    if kind == "norm":
        return _full({**c, "tokens": _log_int(rng, 1, 32768)})
    c.update(block=rng.choice([16, 16, 32, 64]), shuffled=rng.random() < 0.7)
    if kind == "plan":
        batch = _log_int(rng, 1, 1024)
        new = _log_int(rng, 1, max(1, min(8192, 131072 // batch)))
        return _full({**c, "batch": batch, "new_lo": rng.randint(0, new), "new": new, "ctx_lo": 0, "ctx": rng.randint(1, 8000)})
    batch = _log_int(rng, 1, 24)
    if kind in ("append", "latent_rows"):
        c.update(batch=batch, new=_log_int(rng, 1, max(1, 32768 // batch)), ctx_lo=0, ctx=rng.randint(1, 4000))
        if kind == "latent_rows":
            c.update(interleaved=rng.random() < 0.6, anchor=rng.random() < 0.3)
        return _full(c)
    ctx, heads_q = _log_int(rng, 64, 131072), rng.choice([16, 16, 32, 64, 128, 20, 40, 96])
    n = _log_int(rng, 1, 8)
    batch = max(1, min(batch, int(500000 / ctx * min(1.0, 128 / (n * heads_q)))))
    ctx = min(ctx, int(500000 * min(1.0, 128 / (n * heads_q))) // batch)
    return _full({**c, "batch": batch, "n": n, "heads_q": heads_q, "ctx_lo": max(1, ctx // rng.randint(1, 6)), "ctx": ctx, "anchor": rng.random() < 0.3})


# ------------------------------------------------------------------------------------------------ inputs
def _lens(c):
    r = random.Random(c["lens_seed"])
    return [r.randint(c["ctx_lo"], c["ctx"]) for _ in range(c["batch"])]


def _news(c):
    """New tokens of each request of a plan."""
    r = random.Random(c["lens_seed"] + 1000)
    return [r.randint(c["new_lo"], c["new"]) for _ in range(c["batch"])]


def _table(lens, block, shuffled, seed):
    """Block table int32 [batch][blocks of the longest] and the number of blocks of the pool."""
    need = torch.tensor([max(1, -(-n // block)) for n in lens])
    total = int(need.sum())
    perm = torch.randperm(total, generator=torch.Generator().manual_seed(seed)) if shuffled else torch.arange(total)
    table = torch.zeros(len(lens), int(need.max()), dtype=torch.int64)
    table[torch.arange(table.shape[1])[None, :] < need[:, None]] = perm
    return table.to(torch.int32).cuda(), total


def _rotary_inputs(s, tokens, seed, pairs, axes=1, side=16):
    """Positions int32 [axes][tokens] behind a random offset (a run of text, or frames of side x side image patches), the table of cosines
    and sines float32 [positions][pairs cos, pairs sin], and the axis of each pair of channels."""
    t = torch.arange(tokens, device="cuda") + random.Random(seed).randint(0, 999)
    p = t[None] if axes == 1 else torch.stack((t // (side * side), t // side % side + t // (side * side), t % side + t // (side * side)))
    s["positions"] = p.to(torch.int32).contiguous()
    freq = 500000.0 ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
    angle = torch.arange(tokens + 1100, dtype=torch.float64, device="cuda")[:, None] * freq
    s["table"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    s["axis"] = [a for a, n in enumerate(SECTIONS[axes]) for _ in range(n)] if pairs == 64 else [0] * pairs
    s["axis_gpu"] = torch.tensor(s["axis"], device="cuda")


def _weights(g, *shape):
    """A norm's weights, BF16."""
    return (1.0 + 0.3 * torch.randn(*shape, generator=g, device="cuda")).to(torch.bfloat16)


def _quantise(x):
    """8-bit codes, scale and zero point of rows of 128 FP32 values."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    span = hi - lo
    flat = span < 2.0 ** -100
    inv = torch.where(flat, 0.0, 255.0 / span)
    return ((x - lo) * inv).round().to(torch.uint8), torch.cat((torch.where(flat, 0.0, span / 255.0), lo), -1)


def _pack(nib):
    return nib[..., 0::2] | (nib[..., 1::2] << 4)


def _empty_planes(*lead):
    return [torch.zeros(*lead, 64, dtype=torch.uint8, device="cuda"), torch.zeros(*lead, 64, dtype=torch.uint8, device="cuda"),
            torch.zeros(*lead, 2, device="cuda")]


def _prepare_plan(c, s, seed):
    lens, block = _lens(c), c["block"]
    news = [a + n for a, n in zip(lens, _news(c))]
    held, wanted = [-(-n // block) for n in lens], [-(-n // block) for n in news]
    pool = sum(wanted) + 7        # the blocks of all, and a few that stay free
    r = random.Random(seed)
    order = list(range(pool))
    r.shuffle(order)
    table = torch.zeros(c["batch"], max(wanted) + 1, dtype=torch.int64)
    used = torch.arange(table.shape[1])[None, :] < torch.tensor(held)[:, None]
    table[used] = torch.tensor(order[:sum(held)], dtype=torch.int64)
    free, head = order[sum(held):], r.randrange(pool)
    ring = torch.full((pool,), -1, dtype=torch.int64)
    ring[(torch.arange(len(free)) + head) % pool] = torch.tensor(free, dtype=torch.int64)
    s["blocks"], s["ring"] = table.to(torch.int32).cuda(), ring.to(torch.int32).cuda()
    s["state"] = torch.tensor([head, len(free), 0, 0], dtype=torch.int32, device="cuda")
    s["old"], s["new"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, news))
    s["rows"] = max(1, sum(_news(c)) + 5)      # (a few rows of padding behind the last token)
    if own:
        import paper_2607_01831_b200 as lynx
        s["geo"] = lynx.Geometry(8, 8, block, pool, table.shape[1])
        s["pool"] = lynx.BlockPool(s["ring"], s["state"])


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "plan":
        _prepare_plan(c, s, seed)
        return s
    if c["kind"] in ("norm", "append"):     # what a fused projection leaves: views [tokens][heads][128] of one buffer
        tokens = c["tokens"] if c["kind"] == "norm" else c["batch"] * c["new"]
        hq, h = c["heads"] * c["group"], c["heads"]
        x = torch.randn(tokens, hq + 2 * h, D, generator=g, device="cuda")
        x[:, hq:, ::43] *= 10.0
        x = x.to(torch.bfloat16)
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
        s["wq"], s["wk"] = _weights(g, D), _weights(g, D)
        _rotary_inputs(s, tokens, seed, 64, c["axes"], c["side"])
        if own:
            import paper_2607_01831_b200 as lynx
            s["norm"] = lynx.HeadNorm(s["wq"], s["wk"], EPS)
        if c["kind"] == "norm":
            return s
    lens, block = _lens(c), c["block"]
    if c["kind"] in ("append", "latent_rows"):
        first = lens
        lens = [n + c["new"] for n in lens]
        s["rows"] = c["batch"] * c["new"]
        s["starts"] = torch.tensor(first, dtype=torch.int32, device="cuda")
        s["offsets"] = (torch.arange(c["batch"] + 1, device="cuda") * c["new"]).to(torch.int32)
    s["blocks"], pool = _table(lens, block, c["shuffled"], seed)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    heads = c["heads"] if c["kind"] == "append" else 4
    if c["kind"] in ("append", "latent_rows"):
        at = s["starts"].long()[:, None] + torch.arange(c["new"], device="cuda")
        s["slots"] = (s["blocks"].long().gather(1, at // block) * block + at % block).reshape(-1).contiguous()
        s["planes"] = [_empty_planes(pool, heads, block) for _ in range(2 if c["kind"] == "append" else 1)]
    if c["kind"] == "latent_rows":          # a projection's output: a latent and a rotary key a token
        x = torch.randn(s["rows"], LATENT + ROPE, generator=g, device="cuda")
        x[:, ::71] *= 6.0
        x = x.to(torch.bfloat16)
        s["c"], s["kr"], s["wc"] = x[:, :LATENT], x[:, LATENT:], _weights(g, LATENT)
        s["pages"] = torch.zeros(pool, block, ROPE, dtype=torch.bfloat16, device="cuda")
        _rotary_inputs(s, s["rows"], seed, ROPE // 2)
    if c["kind"] == "latent":
        p = _empty_planes(pool, 4, block)
        scale = torch.exp(0.5 * torch.randn(4, 1, D, generator=g, device="cuda"))
        step = max(1, (1 << 24) // (LATENT * block))
        for i in range(0, pool, step):
            n = min(step, pool - i)
            code, p[2][i:i + n] = _quantise((torch.randn(n, 4, block, D, generator=g, device="cuda") * scale).to(torch.bfloat16).float())
            p[0][i:i + n], p[1][i:i + n] = _pack(code >> 4), _pack(code & 15)
        s["planes"] = [p]
        s["pages"] = torch.randn(pool, block, ROPE, generator=g, device="cuda").to(torch.bfloat16)
        s["q"] = torch.randn(c["batch"], c["n"], c["heads_q"], LATENT, generator=g, device="cuda").to(torch.bfloat16)
        s["qr"] = torch.randn(c["batch"], c["n"], c["heads_q"], ROPE, generator=g, device="cuda").to(torch.bfloat16)
    if own:
        import paper_2607_01831_b200 as lynx
        hq = {"append": heads * c.get("group", 1), "latent_rows": heads}.get(c["kind"], c.get("heads_q"))
        s["geo"] = lynx.Geometry(hq, heads, block, pool, s["blocks"].shape[1])
        s["P"] = [lynx.Planes(*p) for p in s["planes"]]
        if c["kind"] == "latent":
            s["ws"] = lynx.make_latent_workspace(s["geo"], c["batch"], c["n"], "cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2607_01831_b200 as lynx
    c = s["case"]
    turn = lynx.Rotary(s["positions"], s["table"], s["axis"], c["interleaved"]) if "table" in s else None
    if c["kind"] == "norm":
        return lynx.norm_rotary(s["q"], s["k"], s["norm"], turn)
    if c["kind"] == "append":
        lynx.cache_append(s["geo"], s["k"], s["v"], s["slots"], *s["P"], rotary=turn, norm=s["norm"])
        return lynx.cache_read(s["geo"], *s["P"], s["blocks"], s["starts"], s["offsets"], s["rows"])
    if c["kind"] == "plan":
        got = lynx.plan_blocks(s["geo"], s["pool"], s["blocks"], s["old"], s["new"], s["rows"])
        back = lynx.plan_blocks(s["geo"], s["pool"], s["blocks"], s["new"], s["old"], 0)
        return got.lens, got.offsets, got.slots, got.positions, back.lens, s["blocks"], s["ring"], s["state"][:2]
    if c["kind"] == "latent_rows":
        lynx.latent_append(s["geo"], s["c"], s["kr"], s["slots"], s["P"][0], s["pages"], weight=s["wc"], eps=EPS, rotary=turn)
        return lynx.latent_read(s["geo"], s["P"][0], s["pages"], s["blocks"], s["starts"], s["offsets"], s["rows"], anchor_only=c["anchor"])
    return lynx.latent_attention(s["geo"], s["q"], s["qr"], s["P"][0], s["pages"], s["blocks"], s["lens"], s["ws"], causal=True,
                                 anchor_only=c["anchor"])


def _normed(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _turned(s, x):
    """x [tokens][heads][2 pairs] FP32 by the positions' angles: pairs of channels (i, i + pairs), or (2 i, 2 i + 1)."""
    n = s["table"].shape[1] // 2
    at = s["positions"].long()[s["axis_gpu"]].t()                           # [tokens][pairs]
    pair = torch.arange(n, device=x.device)
    cos, sin = s["table"][at, pair][:, None], s["table"][at, n + pair][:, None]
    if s["case"]["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x[..., :n], x[..., n:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _values(planes, at, anchor):
    """FP32 values of the rows `at` (an index) of quantised planes: the full codes', or the middle of the Anchor's buckets."""
    a, r, meta = planes[0][at], planes[1][at], planes[2][at]
    a = torch.stack((a & 15, a >> 4), -1).flatten(-2).float()
    low = 8.0 if anchor else torch.stack((r & 15, r >> 4), -1).flatten(-2).float()
    return meta[..., 1:] + meta[..., :1] * (16.0 * a + low)


def _plan(s, old, new, rows):
    """Blocks for the lengths `new` of requests that have `old` tokens: the table, the ring of free blocks and its state are brought up to
    date.  (lengths, offsets, slots and positions of the new tokens)"""
    block, pool = s["case"]["block"], s["ring"].shape[0]
    old, new = old.long(), new.long()
    have, want = -(-old // block), -(-new // block)
    need, give = (want - have).clamp(min=0), (have - want).clamp(min=0)
    head, count = s["state"][0].long(), s["state"][1].long()
    incl = need.cumsum(0)
    fits = (need == 0) | (incl <= count)
    took = torch.where(fits, need, 0)
    column = torch.arange(s["blocks"].shape[1], device="cuda")[None]
    k = column - have[:, None]
    fresh = s["ring"][((head + (incl - need)[:, None] + k) % pool)]
    grown = torch.where((k >= 0) & (k < took[:, None]), fresh, s["blocks"])
    k = column - want[:, None]
    freed = (k >= 0) & (k < give[:, None])
    place = (head + count + (give.cumsum(0) - give)[:, None] + k) % pool
    s["ring"][place[freed]] = s["blocks"][freed]
    s["blocks"].copy_(grown)
    s["state"][0] = (head + took.sum()) % pool
    s["state"][1] = count - took.sum() + give.sum()
    fresh_tokens = (new - old).clamp(min=0)
    offsets = torch.nn.functional.pad(fresh_tokens.cumsum(0), (1, 0))
    row = torch.arange(rows, device="cuda")
    seq = (torch.searchsorted(offsets, row, right=True) - 1).clamp(max=old.shape[0] - 1)
    live = row < offsets[-1]
    token = torch.where(live, old[seq] + row - offsets[seq], 0)
    slot = s["blocks"].long()[seq, token // block] * block + token % block
    return torch.where(fits, new, old).int(), offsets.int(), torch.where(live & fits[seq], slot, -1), token.int()


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "norm":
        return tuple(_turned(s, _normed(s[x].float(), s["w" + x])).to(torch.bfloat16) for x in "qk")
    if c["kind"] == "plan":
        got = _plan(s, s["old"], s["new"], s["rows"])
        table = s["blocks"]
        back = _plan(s, s["new"], s["old"], 0)
        return *got, back[0], table, s["ring"], s["state"][:2]
    block = c["block"]
    if c["kind"] in ("append", "latent_rows"):
        if c["kind"] == "append":
            sources = [_turned(s, _normed(s["k"].float(), s["wk"])), s["v"].float()]
        else:
            sources = [_normed(s["c"].float(), s["wc"]).unflatten(1, (4, D))]
            s["pages"].flatten(0, 1)[s["slots"]] = _turned(s, s["kr"].float()[:, None])[:, 0].to(torch.bfloat16)
        for x, p in zip(sources, s["planes"]):
            code, meta = _quantise(x)
            at = s["slots"] // block, slice(None), s["slots"] % block
            p[0][at], p[1][at], p[2][at] = _pack(code >> 4), _pack(code & 15), meta
        row = torch.arange(s["rows"], device="cuda")
        seq = row // c["new"]
        token = s["starts"].long()[seq] + row - seq * c["new"]
        at = s["blocks"].long()[seq, token // block], slice(None), token % block
        out = [_values(p, at, c.get("anchor", False)).to(torch.bfloat16) for p in s["planes"]]
        if c["kind"] == "append":
            return tuple(out)
        return out[0].flatten(1), s["pages"][at[0], at[2]]
    # attention of the queries over the latents (padded to the longest): keys of 512 + 64 channels, values of 512
    B, n, h = c["batch"], c["n"], c["heads_q"]
    ids = s["blocks"].long()
    V = _values(s["planes"][0], ids, c["anchor"]).transpose(2, 3).flatten(3).flatten(1, 2)         # [B][tokens][512]
    scores = s["q"].float().flatten(1, 2) @ V.transpose(1, 2)
    scores += s["qr"].float().flatten(1, 2) @ s["pages"][ids].float().flatten(1, 2).transpose(1, 2)
    scores *= 192 ** -0.5
    sees = s["lens"][:, None] - n + 1 + torch.arange(n, device="cuda")                               # tokens that position j sees
    scores.masked_fill_(torch.arange(V.shape[1], device="cuda") >= sees.repeat_interleave(h, 1)[:, :, None], -math.inf)
    scores = scores.sub_(scores.amax(2, keepdim=True)).exp_()
    scores.nan_to_num_(nan=0.0)                                                                      # (a position that sees nothing)
    out = scores @ V.masked_fill_((torch.arange(V.shape[1], device="cuda") >= s["lens"][:, None])[:, :, None], 0.0)
    out /= scores.sum(2, keepdim=True).clamp_(min=1e-30)
    return out.view(B, n, h, LATENT).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ accounting
def work(c):
    """Bytes of a row of 128 values: 256 in BF16, 64 per nibble plane, 8 of scale and zero point."""
    if c["kind"] == "plan":
        lens, news, block = _lens(c), _news(c), c["block"]
        fresh, blocks = sum(news), sum(-(-(a + n) // block) - -(-a // block) for a, n in zip(lens, news))
        # lengths in, lengths and offsets out, a slot and a position a token, and a block taken and given back: read and written, twice
        return {"bytes": c["batch"] * 2 * 16 + fresh * 12 + blocks * 16, "flops": fresh * 4}
    if c["kind"] in ("norm", "append"):
        h, tokens = c["heads"], c["tokens"] if c["kind"] == "norm" else c["batch"] * c["new"]
        places = tokens if c["axes"] == 1 else min(tokens, 2 * c["side"] + 3 * (tokens // c["side"] ** 2 + 1))
        more = tokens * c["axes"] * 4 + places * 512
        if c["kind"] == "norm":
            return {"bytes": tokens * h * (c["group"] + 1) * 512 + more, "flops": tokens * h * (c["group"] + 1) * 7 * D}
        return {"bytes": 2 * tokens * h * (256 + 2 * 136 + 256) + more, "flops": 2 * tokens * h * 8 * D}
    row = 72 if c["anchor"] else 136
    if c["kind"] == "latent_rows":
        tokens = c["batch"] * c["new"]
        return {"bytes": tokens * (2 * 1152 + 4 * (136 + row) + 2 * 128 + 256 + 4), "flops": tokens * 10 * LATENT}
    tokens, rows = sum(_lens(c)), c["n"] * c["heads_q"]
    return {"bytes": tokens * (4 * row + 128) + c["batch"] * rows * (1152 + 1024), "flops": 2 * tokens * rows * (2 * LATENT + ROPE)}


# ------------------------------------------------------------------------------------------------ 64-bit results
def exact(case, seed):
    """What run() returns, in 64 bits.  (A plan's outputs are whole numbers: nothing is rounded.)"""
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "plan":
        return None

    def unit(x, w):
        x = x.to(f64)
        return x / ((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.to(f64)

    def spun(x):
        """A pair as a complex number, times cos + i sin."""
        n = s["table"].shape[1] // 2
        at = torch.stack([s["positions"][a] for a in s["axis"]], 1).long()
        turn = torch.complex(s["table"].to(f64).gather(0, at), s["table"].to(f64)[:, n:].gather(0, at))[:, None, :]
        pairs = x.unflatten(2, (n, 2)) if c["interleaved"] else x.unflatten(2, (2, n)).transpose(2, 3)
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        return y.flatten(2) if c["interleaved"] else y.transpose(2, 3).flatten(2)

    if c["kind"] == "norm":
        return spun(unit(s["q"], s["wq"])), spun(unit(s["k"], s["wk"]))

    def coded(x, anchor=False):
        zero = x.min(2, keepdim=True).values
        step = (x.max(2, keepdim=True).values - zero) / 255
        code = torch.round((x - zero) / step)
        return zero + step * (torch.floor(code / 16) * 16 + 8 if anchor else code)

    if c["kind"] == "append":
        return coded(spun(unit(s["k"], s["wk"]))), coded(s["v"].to(f64))
    if c["kind"] == "latent_rows":
        return coded(unit(s["c"], s["wc"]).unflatten(1, (4, D)), c["anchor"]).flatten(1), spun(s["kr"].to(f64)[:, None])[:, 0]
    out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
    for b, length in enumerate(_lens(c)):
        ids = s["blocks"][b, :(length - 1) // c["block"] + 1].long()
        a, r = (p.index_select(0, ids).to(torch.int32) for p in s["planes"][0][:2])
        m = s["planes"][0][2].index_select(0, ids).to(f64)
        level = torch.empty(*a.shape[:-1], D, dtype=f64, device="cuda")
        level[..., 0::2] = (a % 16) * 16 + (8 if c["anchor"] else r % 16)
        level[..., 1::2] = (a // 16) * 16 + (8 if c["anchor"] else r // 16)
        level.mul_(m[..., :1]).add_(m[..., 1:])
        latents = level.permute(0, 2, 1, 3).reshape(-1, LATENT)[:length]
        keys = torch.cat((latents, s["pages"].index_select(0, ids).to(f64).reshape(-1, ROPE)[:length]), 1)
        for j in range(c["n"]):
            count = length - c["n"] + j + 1
            if count > 0:
                x = torch.cat((s["q"][b, j], s["qr"][b, j]), 1).to(f64)
                out[b, j] = (x @ keys[:count].T / math.sqrt(192.0)).softmax(1) @ latents[:count]
    return out
