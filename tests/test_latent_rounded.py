"""The reference and the bounds of tests/latent_rounded.py: FP16 rounding against numpy's, values against the kernel's operations one by one, and what the bounds turn away."""
import math

import numpy as np
import pytest
import torch

import latent_rounded as ref

A = 192 ** -0.5


def _sequence(tokens, seed):
    """Codes [T][4][128], scalars [T][4][2] and rotary keys [T][64] of latents with channels of different sizes."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, 4, 128, generator=g) * torch.exp(0.7 * torch.randn(4, 128, generator=g))
    lo, hi = x.amin(2), x.amax(2)
    scale = (hi - lo) / 255
    return torch.round((x - lo[..., None]) / scale[..., None]), torch.stack((scale, lo), 2), torch.randn(tokens, 64, generator=g).to(torch.bfloat16)


def test_fp16_is_rounded_once():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(100000, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-30, 15, (100000,), generator=g).double())
    ties = torch.tensor([1 + 2.0 ** -11, 1 + 3 * 2.0 ** -11, 2.0 ** -25, 3 * 2.0 ** -25, 2.0 ** -25 + 2.0 ** -60, 1 + 2.0 ** -11 + 2.0 ** -40, 0.0, -0.0, 2.0 ** -26], dtype=torch.float64)
    for v in (x, ties, -ties):
        assert np.array_equal(ref.to_fp16(v).numpy(), v.numpy().astype(np.float16).astype(np.float64))


@pytest.mark.parametrize("anchor", [False, True])
def test_values_are_the_kernels_operations(anchor):
    """numpy's FP16 and FP32, an operation at a time, for some tokens of a sequence whose tiles have different powers of two."""
    code, meta, _ = _sequence(300, 1)
    meta[128:256] *= 2.0 ** 9
    meta[200, 1] *= 2.0 ** 8
    meta[270] = 0
    got = ref.rounded(code, meta, anchor)
    for t in (0, 127, 128, 199, 200, 255, 256, 270, 299):
        rows = meta[t // 128 * 128:t // 128 * 128 + 128].numpy()
        big = max(np.float32(abs(np.float32(128 * float(s) + float(z)))) + np.float32(128) * abs(s) for s, z in rows.reshape(-1, 2))
        e = math.frexp(big)[1] - 1 - 14
        assert 2 ** 14 <= big * 2.0 ** -e < 2 ** 15
        for g in range(4):
            s, z = np.float32(meta[t, g, 0].numpy() * 2.0 ** -e), np.float32(meta[t, g, 1].numpy() * 2.0 ** -e)
            mid = np.float16(np.float32(128.0 * float(s) + float(z)))
            c = code[t, g].numpy()
            c = np.floor(c / 16) * 16 + 8 if anchor else c
            want = ((c - 128) * float(np.float16(s)) + float(mid)).astype(np.float16).astype(np.float64) * 2.0 ** e
            assert np.array_equal(got[t, 128 * g:128 * g + 128].numpy(), want)


@pytest.mark.parametrize("tokens,n", [(16, 1), (300, 4), (2500, 1), (8000, 1)])
@pytest.mark.parametrize("anchor", [False, True])
@pytest.mark.parametrize("step", [2.0 ** -8, 2.0 ** -24])
def test_wrong_outputs_are_turned_away(tokens, n, anchor, step):
    g = torch.Generator().manual_seed(tokens + n)
    code, meta, keys = _sequence(tokens, tokens)
    v = ref.rounded(code, meta, anchor)
    counts = [tokens - n + 1 + j for j in range(n)]
    q, qr = ref.pointed_queries(v, keys, counts, 16, A, g)
    tiles = -(-tokens // 128)

    def far(values, rope, scale=1.0, fewer=0, swap=False, size=1.0, mean=False, loses=slice(0, 0)):
        """The worst error over all positions where the outputs are another calculation's."""
        most, most_out = 0.0, 0.0
        for j, count in enumerate(counts):
            m = max(1, count - fewer)
            out, lse, w = ref.attention(values[:m], rope[:m], q[j], qr[j], A * scale)
            if mean:
                out = values[:m].mean(0).expand(out.shape)
            if loses.stop:
                out = out - w[:, loses] @ values[:m][loses]
            if swap:
                out = out.view(16, 256, 2).flip(2).flatten(1)
            out = out * size
            out = out.to(torch.bfloat16 if step == 2.0 ** -8 else torch.float32)
            args = v[:count], keys[:count], q[j], qr[j], A, step, tiles
            most, most_out = max(most, ref.worst(out, lse, *args)), max(most_out, ref.worst(out, None, *args))
        return most, most_out

    right, _ = far(v, keys)
    assert right <= 1.0
    wrong = {
        "zeros": far(v, keys, size=0.0)[1],
        "5 % too large": far(v, keys, size=1.05)[1],
        "2 % too large": far(v, keys, size=1.02)[1],
        "no rotary part": far(v, torch.zeros_like(keys))[1],
        "a scale 5 % off": far(v, keys, scale=1.05)[1],
        "channels swapped": far(v, keys, swap=True)[1],
        "the mean": far(v, keys, mean=True)[1],
        "one token too few": far(v, keys, fewer=1)[0],
        "16 tokens too few": far(v, keys, fewer=16)[0],
        "the other state of the planes": far(ref.rounded(code, meta, not anchor), keys)[1],
        "a token lost from the sum": far(v, keys, loses=slice(counts[0] - 1, counts[0]))[1],
    }
    assert min(wrong.values()) > 2.0, {k: x for k, x in wrong.items() if x <= 2.0}


@pytest.mark.parametrize("units,right", [(1, True), (8, False)])
def test_weights_roundings_are_what_is_allowed(units, right):
    """Each weight off by a half step of FP16, all for the worse of an output's sign; eight times as much is too far off."""
    code, meta, keys = _sequence(700, 5)
    v = ref.rounded(code, meta)
    q, qr = ref.pointed_queries(v, keys, [700], 16, A, torch.Generator().manual_seed(6))
    out, lse, w = ref.attention(v, keys, q[0], qr[0], A)
    out = out + units * ref.U * out.sign() * (w @ v.abs()) * (1 - 2.0 ** -10)
    assert (ref.worst(out.float(), lse, v, keys, q[0], qr[0], A, 2.0 ** -24, 6) <= 1.0) is right
