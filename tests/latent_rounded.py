"""What attention over quantised latents is to give, with the rounding of its values made as the kernel makes it, and bounds for what is left.

Values.  A code c of a row with the scalars (scale, zero) stands for zero + scale c = middle + scale (c - 128).  Relative to a power of two 2^e of its tile (tokens [128 i,
128 i + 128) of the sequence: the largest value that one of its rows could hold comes to [2^14, 2^15)), scale and middle are rounded to FP16, then middle + scale (c - 128) is.
All of that can be repeated exactly, so that no bound needs to hold for it.
Scores.  The products of a score are exact; of their sums, a step of 16 terms may lose 2^-23 of the largest partial sum for each of its terms that is not zero and for the sum
before, and a partial sum is at most S = sum |q v| over latent and rotary part: (k + 36) 2^-23 S for queries with k values that are not zero, in 36 steps.  Behind them a
few FP32 operations, on at most 2^2 (1 + |score|) in the exponent of two: 2^-20 (1 + |score|).  With D both of a token, its weight is off by a factor within e^+-D: by `off`.
Weights are FP16 in the second product: U = 2^-11 of each, or 2^-27 of the row's largest (which is 2^2 or more) below FP16's normal range, but no more than the weight itself.  Its sums: 17 terms a step, 2^-23 of a partial sum
each, 8 steps a tile and as many tiles as a CTA's range has; the sum of weights is FP32, 4 additions a tile and thread; the CTAs' results are joined in FP32 (2^-20 covers that, and the
references' changes).
Outputs: half a step of their type (2^-8, or 2^-24)."""
import math

import torch

U = 2.0 ** -11
TILE = 128


def to_fp16(x):
    """Float64 values rounded once to FP16's (ties to even), as float64."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), torch.clamp(e - 1, min=-14) - 10)
    return torch.round(x / step) * step


def rounded(code, meta, anchor=False):
    """Values float64 [T][512] of codes [T][4][128] and float32 scalars [T][4][2] of one sequence, as the products have them."""
    T = code.shape[0]
    c = code.double()
    if anchor:
        c = torch.floor(c / 16) * 16 + 8
    scale, zero = meta[..., 0].float(), meta[..., 1].float()
    most = ((128 * scale.double() + zero.double()).float().abs() + 128 * scale.abs()).amax(1)
    tiles = torch.nn.functional.pad(most, (0, -T % TILE)).view(-1, TILE).amax(1)
    _, e = torch.frexp(tiles)                     # (2^(e - 1) <= largest < 2^e)
    e = torch.where(tiles > 0, torch.clamp(e - 15, -80, 113), 0).repeat_interleave(TILE)[:T, None]
    two = torch.ldexp(torch.ones(T, 1, dtype=torch.float64, device=code.device), e)
    s = scale.double() / two
    mid = (128 * s + zero.double() / two).float().double()
    return (to_fp16(to_fp16(mid)[..., None] + (c - 128) * to_fp16(s)[..., None]) * two[..., None]).flatten(1)


def attention(v, keys, q, qr, a):
    """Float64: outputs [R][512], log-sum-exps [R] and weights [R][T] of rows q [R][512], qr [R][64] over values v [T][512] and rotary keys [T][64]."""
    s = a * (q.double() @ v.T + qr.double() @ keys.double().T)
    w = s.softmax(1)
    return w @ v, s.logsumexp(1), w


def bounds(v, keys, q, qr, a, want, lse, w, step, tiles):
    """For outputs [R][512] and log-sum-exps [R]; step: half a step of the outputs' type; tiles: of a CTA's range."""
    terms = (q != 0).sum(1, keepdim=True) + (qr != 0).sum(1, keepdim=True) + 36
    log_w = w.clamp(min=1e-300).log()
    S = a * (q.double().abs() @ v.abs().T + qr.double().abs() @ keys.double().abs().T)
    D = terms * 2.0 ** -23 * S + 2.0 ** -20 * (1 + lse[:, None].abs() + log_w.abs())
    off = torch.where((w > 0) & (log_w + D > -45), torch.expm1(D.clamp(max=60)) * w, 0)      # (what is smaller by e^-45 is none)
    off_sum = off.sum(1, keepdim=True)
    sums = 17 * 8 * tiles * 2.0 ** -23 + (4 * tiles + 16) * 2.0 ** -24 + 2.0 ** -20
    tail = torch.minimum(2.0 ** -27 * w.amax(1, keepdim=True), w + off) @ v.abs()
    usual = w @ v.abs()
    bound = (off @ v.abs() + off_sum * usual) * (1 + 2 * off_sum) + (U + sums) * usual + tail + step * want.abs()
    return bound, off_sum[:, 0] * (1 + off_sum[:, 0]) + sums + 2.0 ** -22 * lse.abs()


def _as_multiple(off, bound):
    return float(torch.where(off == 0, 0.0, off / bound).nan_to_num(math.inf).max())


def worst(got, gl, v, keys, q, qr, a, step, tiles):
    """The largest error of outputs and log-sum-exps (or None) as a multiple of its bound: right at up to 1.  No number is infinitely wrong."""
    want, lse, w = attention(v, keys, q, qr, a)
    bound, lb = bounds(v, keys, q, qr, a, want, lse, w, step, tiles)
    far = _as_multiple((got.double() - want).abs(), bound)
    return far if gl is None else max(far, _as_multiple((gl.double() - lse).abs(), lb))


def pointed_queries(v, keys, counts, heads, a, g, positive=False):
    """Rows [len(counts)][heads] that each look for one token: eight channels of it, two of each 128, and two of its rotary key, so that it takes about half of the weight.  Of positions that see `counts` tokens
    each: the last that they see, the first that they do not see, the ends of tiles, others by chance.  positive: latent parts without negative values, of tokens that have
    channels above zero."""
    T = v.shape[0]
    q, qr = torch.zeros(len(counts), heads, 512), torch.zeros(len(counts), heads, 64)
    v, keys = v.cpu(), keys.double().cpu()
    size_of = (lambda x: x) if positive else torch.abs
    for j, n in enumerate(counts):
        for h in range(heads):
            chance = int(torch.randint(max(n, 1), (1,), generator=g))
            t = min(max((n - 1, n, 0, chance, 127, 128, chance, n - 2)[h % 8], 0), T - 1)
            while positive and v[t].amax() <= 0:
                t -= 1
            at = torch.cat([128 * i + size_of(v[t, 128 * i:128 * i + 128]).topk(24).indices[torch.randperm(24, generator=g)[:2]] for i in range(4)])
            rope = keys[t].abs().topk(16).indices[torch.randperm(16, generator=g)[:2]]
            size = float(v[t, at].abs().sum() + keys[t, rope].abs().sum())
            strength = (math.log(max(n, 1)) + 2) / (a * size) if size else 0.0
            q[j, h, at] = (v[t, at].sign() * strength).float()
            qr[j, h, rope] = (keys[t, rope].sign() * strength).float()
    return q.to(torch.bfloat16), qr.to(torch.bfloat16)
