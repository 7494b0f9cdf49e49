"""Timed cases of the operators around a quantised cache: rotary positions, writing tokens into the cache and reading them
back, and attention of a tree of drafted tokens over it.

A step of a decode node that drafts trees: the nodes' queries and keys get their rotary positions, the nodes attend to the
quantised prefix and to their ancestors, and the accepted nodes' keys and values are quantised into the cache.  Prompts and
plain decode steps are rotated and quantised in one go; ranges of the cache go back to BF16 for an engine that wants them so.
Shapes are those of the repository's other workloads: 8 KV heads of 128 channels with 32 or 64 query heads, contexts
up to 131072 tokens, blocks of 16 tokens (32 and 64 among the drawn cases), uniform or ragged batches.

`own` false: elementary torch operations in 32 bits.  `own` true: the library's entry points.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
SECTIONS = {1: (64,), 3: (16, 24, 24)}    # rotary pairs per axis: positions of text, or time, height and width


def listed():
    cases = [
        # Rotary positions of one step's tree nodes: 4 sequences x 7 nodes, positions of text.
        dict(name="rotary_nodes_28", kind="rotary", tokens=28, axes=1),
        # Rotary positions of a long prompt made of images: time, height and width, 64 query heads.
        dict(name="rotary_images_32k", kind="rotary", tokens=32768, axes=3, group=8, side=48),
        # A decode step of 16 ragged sequences: one token each, rotated and quantised into its slot, and read back.
        dict(name="append_decode_16", kind="append", batch=16, new=1, ctx_lo=500, ctx=4000, rotate=True),
        # A prompt of 32768 tokens with image positions, rotated and quantised into scattered blocks, and read back.
        dict(name="append_prompt_32k", kind="append", batch=1, new=32768, ctx_lo=0, ctx=0, axes=3, rotate=True, side=32,
             values="outlier"),
        # The last 100 tokens (an odd start) of 4 sequences, back to BF16.
        dict(name="read_tail_4x100", kind="read", batch=4, ctx_lo=901, ctx=2001, count=100, values="student_t"),
        # A whole layer of a long context, back to BF16.
        dict(name="read_layer_128k", kind="read", batch=1, ctx_lo=131072, ctx=131072, count=131072, shuffled=False),
        # One token over a short cache: the smallest call.
        dict(name="tree_1_ctx_300", kind="tree", batch=1, n=1, ctx_lo=300, ctx=300),
        # A small tree over a 4096-token context, one layer.
        dict(name="tree_13_ctx_4k", kind="tree", batch=1, n=13, ctx_lo=4096, ctx=4096, values="outlier"),
        # Drafting a tree's next level on the Anchor plane alone, a serving mix of ragged sequences in shuffled blocks.
        dict(name="tree_5_mix_anchor", kind="tree", batch=16, n=5, ctx_lo=8192, ctx=65536, anchor=True, values="student_t"),
        # Verifying trees of 24 nodes in the same mix.
        dict(name="tree_24_mix", kind="tree", batch=16, n=24, ctx_lo=8192, ctx=65536, values="student_t"),
        # A tree of 32 nodes (128 query columns per KV head) over one long context.
        dict(name="tree_32_layer_128k", kind="tree", batch=1, n=32, ctx_lo=131072, ctx=131072, shuffled=False),
        # The largest trees, 64 nodes with 8 query heads per KV head (512 columns), over two long contexts.
        dict(name="tree_64_70b_2x128k", kind="tree", batch=2, n=64, group=8, ctx_lo=131072, ctx=131072, values="outlier"),
    ]
    return [_full(c) for c in cases]


def _full(c):
    """Every option of a case spelt out.  ctx_lo < ctx: ragged lengths, drawn from lens_seed."""
    base = dict(heads=8, group=4, lens_seed=1)
    if c["kind"] in ("rotary", "append"):
        base.update(axes=1, side=16, interleaved=False)
    if c["kind"] != "rotary":
        base.update(batch=1, block=16, shuffled=True, values="lognormal")
    if c["kind"] == "append":
        base.update(rotate=False, nodes=0)
    if c["kind"] in ("read", "tree"):
        base.update(anchor=False)
    return {**base, **c}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    kind = rng.choice(["rotary", "append", "read", "tree", "tree", "tree"])
    c = dict(kind=kind, group=rng.choice([4, 4, 8, 8, 1, 2]), lens_seed=rng.randint(1, 1000))
    if kind in ("rotary", "append"):
        c.update(axes=rng.choice([1, 3]), side=rng.randint(3, 64), interleaved=rng.random() < 0.3)
    if kind == "rotary":
        return _full({**c, "tokens": _log_int(rng, 1, 32768)})
    c.update(block=rng.choice([16, 16, 32, 64]), shuffled=rng.random() < 0.7, values=rng.choice(["lognormal", "student_t", "outlier"]))
    batch = _log_int(rng, 1, 24)
    if kind == "append":
        new = _log_int(rng, 1, max(1, 32768 // batch))
        if new <= 64 and rng.random() < 0.5:      # accepted nodes of a tree, rotated before
            c.update(nodes=rng.randint(new, 64))
        else:
            c.update(rotate=True)
        return _full({**c, "batch": batch, "new": new, "ctx_lo": 0, "ctx": rng.randint(1, 4000)})
    ctx = _log_int(rng, 64, 131072)
    if kind == "read":
        batch = max(1, min(batch, 131072 // ctx))
        return _full({**c, "batch": batch, "ctx_lo": max(1, ctx // rng.randint(1, 6)), "ctx": ctx,
                      "count": max(1, min(ctx, _log_int(rng, 16, 131072))), "anchor": rng.random() < 0.3})
    n = _log_int(rng, 1, 64)
    batch = max(1, min(batch, (600000 if n * c["group"] <= 128 else 262144) // ctx))
    return _full({**c, "batch": batch, "n": n, "ctx_lo": max(1, ctx // rng.randint(1, 6)), "ctx": ctx, "anchor": rng.random() < 0.3})


# ------------------------------------------------------------------------------------------------ inputs
def _lens(c):
    r = random.Random(c["lens_seed"])
    return [r.randint(c["ctx_lo"], c["ctx"]) for _ in range(c["batch"])]


def _ranges(c):
    """(first token, number of tokens) per sequence that a pass writes or reads back."""
    if c["kind"] == "append":
        return [(n, c["new"]) for n in _lens(c)]
    return [(max(0, n - c["count"]), min(n, c["count"])) for n in _lens(c)]


def _table(lens, block, shuffled, seed):
    """Block table int32 [batch][blocks of the longest] and the number of blocks of the pool."""
    need = torch.tensor([max(1, -(-n // block)) for n in lens])
    total = int(need.sum())
    perm = torch.randperm(total, generator=torch.Generator().manual_seed(seed)) if shuffled else torch.arange(total)
    table = torch.zeros(len(lens), int(need.max()), dtype=torch.int64)
    table[torch.arange(table.shape[1])[None, :] < need[:, None]] = perm
    return table.to(torch.int32).cuda(), total


def _positions(c, tokens, seed):
    """Rotary positions int32 [axes][tokens] behind a random offset: a run of text, or frames of side x side image patches."""
    t = torch.arange(tokens, device="cuda") + random.Random(seed).randint(0, 999)
    s = c["side"]
    p = t[None] if c["axes"] == 1 else torch.stack((t // (s * s), t // s % s + t // (s * s), t % s + t // (s * s)))
    return p.to(torch.int32).contiguous()


def _rotary_inputs(c, s, tokens, seed):
    """Positions, the table of cosines and sines float32 [positions][64 cos, 64 sin], and the axis of each pair of channels."""
    s["positions"] = _positions(c, tokens, seed)
    freq = 500000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    angle = torch.arange(tokens + 1100, dtype=torch.float64, device="cuda")[:, None] * freq
    s["table"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    s["axis"] = [a for a, n in enumerate(SECTIONS[c["axes"]]) for _ in range(n)]
    s["axis_gpu"] = torch.tensor(s["axis"], device="cuda")


def _projected(c, g, tokens):
    """What a fused projection leaves: BF16 views q [tokens][Hq][128], k, v [tokens][heads][128] of one buffer."""
    hq, h = c["heads"] * c["group"], c["heads"]
    x = torch.randn(tokens, hq + 2 * h, D, generator=g, device="cuda")
    if c.get("values") == "outlier":
        x[:, hq:, ::43] *= 10.0
    x = x.to(torch.bfloat16)
    return x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]


def _quantise(x):
    """8-bit codes, scale and zero point of rows of 128 FP32 values."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    span = hi - lo
    flat = span < 2.0 ** -100
    inv = torch.where(flat, 0.0, 255.0 / span)
    return ((x - lo) * inv).round().to(torch.uint8), torch.cat((torch.where(flat, 0.0, span / 255.0), lo), -1)


def _pack(nib):
    return nib[..., 0::2] | (nib[..., 1::2] << 4)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "rotary":
        s["q"], s["k"], _ = _projected(c, g, c["tokens"])
        _rotary_inputs(c, s, c["tokens"], seed)
        return s
    lens, block, heads = _lens(c), c["block"], c["heads"]
    if c["kind"] == "append":
        lens = [n + c["new"] for n in lens]
    s["blocks"], pool = _table(lens, block, c["shuffled"], seed)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if c["kind"] in ("append", "read"):
        starts, counts = (torch.tensor(x) for x in zip(*_ranges(c)))
        s["starts"] = starts.to(torch.int32).cuda()
        s["offsets"] = torch.cat((torch.zeros(1, dtype=torch.int64), counts.cumsum(0))).to(torch.int32).cuda()
        s["rows"] = int(counts.sum())
    shape = (pool, heads, block)
    if c["kind"] == "append":
        s["planes"] = [[torch.zeros(*shape, 64, dtype=torch.uint8, device="cuda"), torch.zeros(*shape, 64, dtype=torch.uint8, device="cuda"),
                        torch.zeros(*shape, 2, device="cuda")] for _ in range(2)]
        tokens = c["batch"] * (c["nodes"] or c["new"])
        _, s["k"], s["v"] = _projected(c, g, tokens)
        token = torch.arange(c["new"], device="cuda")
        at = s["starts"].long()[:, None] + token
        s["slots"] = (s["blocks"].long().gather(1, at // block) * block + at % block).reshape(-1).contiguous()
        if c["nodes"]:      # the accepted nodes of each tree
            pick = torch.rand(c["batch"], c["nodes"], generator=g, device="cuda").argsort(1)[:, :c["new"]].sort(1)[0]
            s["accepted"] = (pick + c["nodes"] * torch.arange(c["batch"], device="cuda")[:, None]).reshape(-1).to(torch.int32)
        if c["rotate"]:
            _rotary_inputs(c, s, tokens, seed)
    else:
        s["planes"] = []
        step = max(1, (1 << 24) // (heads * block * D))
        for _ in range(2):
            scale = torch.exp(0.5 * torch.randn(heads, 1, D, generator=g, device="cuda")) if c["values"] == "lognormal" else \
                torch.ones(heads, 1, D, device="cuda")
            if c["values"] == "outlier":      # three channels of 128 ten times the rest
                scale.scatter_(2, torch.rand(heads, D, generator=g, device="cuda").argsort(1)[:, None, :3], 10.0)
            p = [torch.empty(*shape, 64, dtype=torch.uint8, device="cuda"), torch.empty(*shape, 64, dtype=torch.uint8, device="cuda"),
                 torch.empty(*shape, 2, device="cuda")]
            for i in range(0, pool, step):
                n = min(step, pool - i)
                x = torch.randn(n, heads, block, D, generator=g, device="cuda")
                if c["values"] == "student_t":
                    x /= (torch.randn(4, n, heads, block, D, generator=g, device="cuda").square_().sum(0) * 0.25).sqrt_()
                code, p[2][i:i + n] = _quantise((x * scale).to(torch.bfloat16).float())
                p[0][i:i + n], p[1][i:i + n] = _pack(code >> 4), _pack(code & 15)
            s["planes"].append(p)
    if c["kind"] == "tree":
        n = c["n"]
        q, k, v = _projected(c, g, c["batch"] * n)
        s["q"] = q.contiguous().view(c["batch"], n, -1, D)
        s["k"] = k.contiguous().view(c["batch"], n, heads, D)
        s["v"] = v.unflatten(0, (c["batch"], n))     # (a view of the projection's output; q and k come from the rotation)
        r, masks = random.Random(seed), []
        for _ in range(c["batch"]):                  # each node sees itself and its ancestors
            m = []
            for j in range(n):
                m.append((m[r.randint(max(0, j - 6), j - 1)] if j else 0) | (1 << j))
            masks.append([x - (1 << 64) if x >> 63 else x for x in m])
        s["mask"] = torch.tensor(masks, dtype=torch.int64, device="cuda")
    if own:
        import paper_2607_01831_b200 as lynx
        s["geo"] = lynx.Geometry(heads * c["group"], heads, block, pool, s["blocks"].shape[1])
        s["K"], s["V"] = (lynx.Planes(*p) for p in s["planes"])
        if c["kind"] == "tree":
            s["ws"] = lynx.make_tree_workspace(s["geo"], c["batch"], c["n"], "cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2607_01831_b200 as lynx
    c = s["case"]
    turn = lynx.Rotary(s["positions"], s["table"], s["axis"], c["interleaved"]) if "table" in s else None
    if c["kind"] == "rotary":
        return lynx.rotary(s["q"], s["k"], turn)
    if c["kind"] == "append":
        lynx.cache_append(s["geo"], s["k"], s["v"], s["slots"], s["K"], s["V"], rows=s.get("accepted"), rotary=turn)
        return lynx.cache_read(s["geo"], s["K"], s["V"], s["blocks"], s["starts"], s["offsets"], s["rows"])
    if c["kind"] == "read":
        return lynx.cache_read(s["geo"], s["K"], s["V"], s["blocks"], s["starts"], s["offsets"], s["rows"], anchor_only=c["anchor"])
    return lynx.tree_attention(s["geo"], s["q"], s["K"], s["V"], s["blocks"], s["lens"], s["k"], s["v"], s["mask"], s["ws"],
                               anchor_only=c["anchor"])


def _turned(s, x):
    """x [tokens][heads][128] FP32 by the positions' angles: pairs of channels (i, i + 64), or (2 i, 2 i + 1)."""
    at = s["positions"].long()[s["axis_gpu"]].t()                           # [tokens][64]
    pair = torch.arange(64, device=x.device)
    cos, sin = s["table"][at, pair][:, None], s["table"][at, 64 + pair][:, None]
    if s["case"]["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x[..., :64], x[..., 64:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _values(planes, at, anchor):
    """FP32 values of the rows `at` (an index) of quantised planes: the full codes', or the middle of the Anchor's buckets."""
    a, r, meta = planes[0][at], planes[1][at], planes[2][at]
    a = torch.stack((a & 15, a >> 4), -1).flatten(-2).float()
    low = 8.0 if anchor else torch.stack((r & 15, r >> 4), -1).flatten(-2).float()
    return meta[..., 1:] + meta[..., :1] * (16.0 * a + low)


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rotary":
        return _turned(s, s["q"].float()).to(torch.bfloat16), _turned(s, s["k"].float()).to(torch.bfloat16)
    block = c["block"]
    if c["kind"] == "append":
        k, v = s["k"].float(), s["v"].float()
        k = _turned(s, k) if c["rotate"] else k
        k, v = (k[s["accepted"]], v[s["accepted"]]) if c["nodes"] else (k, v)
        for x, p in zip((k, v), s["planes"]):
            code, meta = _quantise(x)
            at = s["slots"] // block, slice(None), s["slots"] % block
            p[0][at], p[1][at], p[2][at] = _pack(code >> 4), _pack(code & 15), meta
    if c["kind"] in ("append", "read"):
        row = torch.arange(s["rows"], device="cuda")
        seq = torch.searchsorted(s["offsets"].long(), row, right=True) - 1
        token = s["starts"].long()[seq] + row - s["offsets"].long()[seq]
        at = s["blocks"].long()[seq, token // block], slice(None), token % block
        return tuple(_values(p, at, c.get("anchor", False)).to(torch.bfloat16) for p in s["planes"])
    # attention of the nodes over the prefix (padded to the longest) and over each other
    B, n, h, grp = c["batch"], c["n"], c["heads"], c["group"]
    q = s["q"].float().view(B, n, h, grp, D).permute(0, 2, 1, 3, 4).reshape(B, h, n * grp, D) / math.sqrt(D)
    K, V = (_values(p, s["blocks"].long(), c["anchor"]).permute(0, 2, 1, 3, 4).reshape(B, h, -1, D) for p in s["planes"])
    scores = q @ K.transpose(2, 3)
    scores.masked_fill_((torch.arange(K.shape[2], device="cuda") >= s["lens"][:, None])[:, None, None], -math.inf)
    k, v = (s[x].float().permute(0, 2, 1, 3) for x in "kv")
    sees = (s["mask"][:, :, None] >> torch.arange(n, device="cuda") & 1).bool().repeat_interleave(grp, 1)[:, None]
    among = (q @ k.transpose(2, 3)).masked_fill_(~sees, -math.inf)
    top = torch.maximum(scores.amax(3, keepdim=True), among.amax(3, keepdim=True))
    scores, among = scores.sub_(top).exp_(), (among - top).exp()
    out = (scores @ V.masked_fill_((torch.arange(V.shape[2], device="cuda") >= s["lens"][:, None])[:, None, :, None], 0.0) + among @ v)
    out /= scores.sum(3, keepdim=True) + among.sum(3, keepdim=True)
    return out.view(B, h, n, grp, D).permute(0, 2, 1, 3, 4).reshape(B, n, h * grp, D).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ accounting
def work(c):
    """Bytes of a row of 128 values: 256 in BF16, 64 per nibble plane, 8 of scale and zero point."""
    h, grp = c["heads"], c["group"]
    if c["kind"] == "rotary":
        t = c["tokens"]
        places = t if c["axes"] == 1 else min(t, 2 * c["side"] + 3 * (t // c["side"] ** 2 + 1))
        return {"bytes": t * h * (grp + 1) * 512 + t * c["axes"] * 4 + places * 512, "flops": t * h * (grp + 1) * 3 * D}
    if c["kind"] == "append":
        rows = 2 * c["batch"] * c["new"] * h            # BF16 in; planes out and in; BF16 out
        places = 0 if not c["rotate"] else c["batch"] * c["new"]
        places = places if c.get("axes", 1) == 1 else min(places, 2 * c["side"] + 3 * (places // c["side"] ** 2 + 1))
        return {"bytes": rows * (256 + 2 * 136 + 256) + places * 512, "flops": rows * 6 * D}
    row = 72 if c["anchor"] else 136
    if c["kind"] == "read":
        rows = 2 * h * sum(n for _, n in _ranges(c))
        return {"bytes": rows * (row + 256), "flops": rows * 2 * D}
    tokens, nodes = h * sum(_lens(c)), h * c["batch"] * c["n"]
    return {"bytes": 2 * tokens * row + nodes * (2 + 2 * grp) * 256, "flops": 4 * (tokens + nodes * c["n"]) * c["n"] * grp * D}


# ------------------------------------------------------------------------------------------------ 64-bit results
def exact(case, seed):
    """What run() returns, in 64 bits."""
    c, s = case, prepare(case, seed)
    f64 = torch.float64

    def spun(x):
        """A pair as a complex number, times cos + i sin."""
        at = torch.stack([s["positions"][a] for a in s["axis"]], 1).long()
        turn = torch.complex(s["table"].to(f64).gather(0, at), s["table"].to(f64)[:, 64:].gather(0, at))[:, None, :]
        x = x.to(f64)
        pairs = x.unflatten(2, (64, 2)) if c["interleaved"] else x.unflatten(2, (2, 64)).transpose(2, 3)
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        return y.flatten(2) if c["interleaved"] else y.transpose(2, 3).flatten(2)

    if c["kind"] == "rotary":
        return spun(s["q"]), spun(s["k"])
    if c["kind"] == "append":
        out = []
        for name in "kv":
            x = spun(s[name]) if name == "k" and c["rotate"] else s[name].to(f64)
            if c["nodes"]:
                x = x.index_select(0, s["accepted"].long())
            zero = x.min(2, keepdim=True).values
            step = (x.max(2, keepdim=True).values - zero) / 255
            out.append(zero + step * torch.round((x - zero) / step))
        return tuple(out)

    def rows(planes, b, first, count):
        """[count][heads][128] of tokens first .. first + count - 1 of sequence b."""
        lo, hi = first // c["block"], (first + count - 1) // c["block"] + 1
        ids = s["blocks"][b, lo:hi].long()
        a, r = (p.index_select(0, ids).to(torch.int32) for p in planes[:2])
        m = planes[2].index_select(0, ids).to(f64)
        level = torch.empty(*a.shape[:-1], D, dtype=f64, device="cuda")
        level[..., 0::2] = (a % 16) * 16 + (8 if c["anchor"] else r % 16)
        level[..., 1::2] = (a // 16) * 16 + (8 if c["anchor"] else r // 16)
        level.mul_(m[..., :1]).add_(m[..., 1:])
        return level.transpose(1, 2).flatten(0, 1)[first - lo * c["block"]:][:count]

    if c["kind"] == "read":
        return tuple(torch.cat([rows(p, b, *span) for b, span in enumerate(_ranges(c))]) for p in s["planes"])
    out = torch.empty(s["q"].shape, dtype=f64, device="cuda")
    n = c["n"]
    bits = torch.tensor([[[(m >> i) & 1 for i in range(n)] for m in ms] for ms in s["mask"].tolist()], device="cuda").bool()
    for b, length in enumerate(_lens(c)):
        keys, values = (torch.cat((rows(p, b, 0, length), s[x][b].to(f64))) for p, x in zip(s["planes"], "kv"))
        allowed = torch.cat((torch.ones(n, length, dtype=torch.bool, device="cuda"), bits[b]), 1)
        for head in range(c["heads"] * c["group"]):
            kv = head // c["group"]
            w = (s["q"][b, :, head].to(f64) @ keys[:, kv].T) * D ** -0.5
            w = torch.where(allowed, w, -math.inf).softmax(1)
            out[b, :, head] = w @ values[:, kv]
    return out
