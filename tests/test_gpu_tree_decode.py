"""The example that decodes with drafted trees: each attention of it against a plain one in 64 bits, and what its cache holds at the end."""
import importlib.util
import os

import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tree_decode.py")
    spec = importlib.util.spec_from_file_location("tree_decode", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _rows(planes, anchor_only):
    def nibbles(p):
        return torch.stack((p & 15, p >> 4), -1).flatten(-2).double()

    code = 16 * nibbles(planes.anchor) + (8 if anchor_only else nibbles(planes.residual))
    return planes.meta[..., 1:].double() + planes.meta[..., :1].double() * code      # [block][head][token][128]


def _checked_attention(real, calls):
    """tree_attention, each of its results compared with a plain evaluation in 64 bits.  Bound: the output's rounding to BF16, 2^-8 of it,
    and (2^-9 + 2 E) A, E = 2^-16 S: A the largest |mid| + 128 |scale| of the values, S the largest |scale| |q|_1 (|mid| + 128 |scale|) of the
    keys (values and weights enter as FP16, scores and sums are FP32)."""
    def attention(geo, q, K, V, blocks, lens, k, v, mask, workspace, anchor_only=False):
        got = real(geo, q, K, V, blocks, lens, k, v, mask, workspace, anchor_only=anchor_only)
        lynx.check(workspace)
        B, n, Hq, _ = q.shape
        group, out, worst = Hq // geo.num_kv_heads, torch.zeros(q.shape, dtype=torch.float64, device=q.device), []
        ks, vs = _rows(K, anchor_only), _rows(V, anchor_only)
        for b in range(B):
            L, at = int(lens[b]), blocks[b].long()
            keys, vals, km, vm = (x[at].transpose(1, 2).flatten(0, 1)[:L].double() for x in (ks, vs, K.meta, V.meta))    # [token][head][..]
            mids = [torch.cat((m[..., 1] + 128 * m[..., 0], m.new_zeros(n, m.shape[1]))) for m in (km, vm)]
            devs = [torch.cat((128 * m[..., 0], x.double().abs().amax(-1))) for m, x in ((km, k[b]), (vm, v[b]))]
            keys, vals = torch.cat((keys, k[b].double())), torch.cat((vals, v[b].double()))
            see = torch.cat((torch.ones(n, L, dtype=torch.bool, device=q.device), (mask[b][:, None] >> torch.arange(n, device=q.device)) & 1 != 0), 1)
            s = torch.einsum("jhd,thd->hjt", q[b].double(), keys.repeat_interleave(group, 1)) / 128 ** 0.5
            p = s.masked_fill(~see, float("-inf")).softmax(-1)
            out[b] = torch.einsum("hjt,thd->jhd", p, vals.repeat_interleave(group, 1))
            S = q[b].double().abs().sum(-1).max() * (mids[0].abs() + devs[0]).max() / 128 ** 0.5
            worst.append((2.0 ** -9 + 2 * 2.0 ** -16 * S) * (mids[1].abs() + devs[1]).max())
        tol = torch.stack(worst)[:, None, None, None] + 2.0 ** -8 * out.abs()
        assert ((got.double() - out).abs() <= tol).all()
        calls.append(n)
        return got
    return attention


@pytest.mark.parametrize("batch,context", [(1, 1), (3, 2), (2, 15), (4, 200)])
def test_decoding_with_trees(batch, context, monkeypatch):
    m = _example()
    calls = []
    monkeypatch.setattr(m.lynx, "tree_attention", _checked_attention(lynx.tree_attention, calls))
    layer = m.Layer(seed=batch)
    prompt = torch.randint(layer.vocab, (batch, context), generator=torch.Generator().manual_seed(context)).cuda()
    d, got, logits, steps = m.decode(layer, prompt, 24)
    assert calls == d.ends * steps
    assert steps <= 24 and d.lens.tolist() == [context - 1 + len(t) for t in got]
    for b in range(batch):      # greedy
        assert len(got[b]) >= 24 and torch.stack(logits[b]).argmax(-1).tolist() == got[b]
    # the cache holds the keys and values of the prompt and of the tokens but the last: half a step of 8 bits and a rounding to BF16 each way,
    # and another where the node's rotated key was rounded before it was quantised
    k, v = d.pages()
    at = 0
    for b in range(batch):
        tokens = torch.cat((prompt[b], torch.tensor(got[b][:-1], dtype=prompt.dtype, device="cuda")))
        _, kx, vx = layer.project(tokens)
        turn = d.table[:len(tokens)].double()
        c, s = turn[:, None, :64], turn[:, None, 64:]
        lo, hi = kx[..., :64].double(), kx[..., 64:].double()
        kx = torch.cat((lo * c - hi * s, hi * c + lo * s), -1)
        for want, have in ((kx, k), (vx.double(), v)):
            have = have[at:at + len(tokens)].double()
            # (the projection's own rounding, 2^-9, may go the other way in a product of another size, and with FP32 sums of 512 terms)
            span = want.amax(-1, keepdim=True) - want.amin(-1, keepdim=True)
            size = want.abs().amax(-1, keepdim=True)
            assert ((have - want).abs() <= span / 510 + size * (4 * 2.0 ** -8)).all()
        at += len(tokens)
