"""Greedy decoding that drafts trees, over a quantised cache: how the entry points around the cache work together.

    python examples/tree_decode.py [--tokens 64] [--batch 4] [--context 4096]

One attention layer with random weights stands for a model.  A step drafts a tree from the last token on the Anchor plane alone, level
by level, verifies all of its nodes in one pass over the full codes, and writes the accepted path into the cache:

    rotary          the nodes' queries and keys, positions by their depth in the tree
    tree_attention  the prefix's planes and the nodes' BF16 keys and values, each node seeing its ancestors
    cache_append    the accepted nodes, quantised into their slots (the prompt, too, rotated on the way)
    cache_read      what the cache holds, as BF16, for an engine that wants pages
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_01831_b200 as lynx  # noqa: E402

# A tree: the level of each node, and its parent.  The root is the last token; it branches into three, and the likelier ones go deeper.
LEVELS = [[-1], [0, 0, 0], [1, 1, 2], [4, 6]]
PARENTS = [p for level in LEVELS for p in level]
DEPTH = [d for d, level in enumerate(LEVELS) for _ in level]
BLOCK = 16


class Layer:
    """An embedding, one attention layer, and the embedding again for the logits."""

    def __init__(self, vocab=1024, dim=512, q_heads=8, kv_heads=2, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device=device) / shape[0] ** 0.5).to(torch.bfloat16)

        self.q_heads, self.kv_heads, self.vocab = q_heads, kv_heads, vocab
        self.embed = torch.randn(vocab, dim, generator=g, device=device).to(torch.bfloat16)
        self.qkv = weight(dim, (q_heads + 2 * kv_heads) * 128)
        self.out = weight(q_heads * 128, dim)
        self.turn = weight(dim, dim)      # (without it a token would always follow itself)

    def project(self, tokens):
        """q, k, v of tokens [T]: views [T][heads][128] of one product."""
        x = (self.embed[tokens] @ self.qkv).view(len(tokens), -1, 128)
        return x.split((self.q_heads, self.kv_heads, self.kv_heads), 1)

    def logits(self, tokens, o):
        """FP32 logits [T][vocab] behind attention's output [T][q_heads * 128]."""
        x = self.embed[tokens].float() @ self.turn.float() + 4.0 * (o.float() @ self.out.float())
        return x @ self.embed.float().t() / x.shape[-1] ** 0.5


class Decoder:
    def __init__(self, layer, batch, capacity, seed=0):
        device = layer.embed.device
        per_seq = (capacity + BLOCK - 1) // BLOCK
        self.layer, self.batch = layer, batch
        self.geo = lynx.Geometry(layer.q_heads, layer.kv_heads, BLOCK, batch * per_seq, per_seq)
        shape = (self.geo.num_blocks, layer.kv_heads, BLOCK)
        self.K, self.V = (lynx.Planes(torch.zeros(*shape, 64, dtype=torch.uint8, device=device),
                                      torch.zeros(*shape, 64, dtype=torch.uint8, device=device), torch.zeros(*shape, 2, device=device))
                          for _ in range(2))
        order = torch.randperm(self.geo.num_blocks, generator=torch.Generator().manual_seed(seed))   # (a pool in use has no order)
        self.blocks = order.to(torch.int32).view(batch, per_seq).to(device)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=device)
        self.table = lynx.rotary_table(capacity, device=device)
        self.ends = [sum(map(len, LEVELS[:d + 1])) for d in range(len(LEVELS))]     # nodes up to each level; all of them are verified
        self.workspace = lynx.make_tree_workspace(self.geo, batch, self.ends[-1], device)      # (for smaller trees, too)
        mask = []
        for j, p in enumerate(PARENTS):                                              # a node sees itself and its ancestors
            mask.append((mask[p] if p >= 0 else 0) | 1 << j)
        self.mask = torch.tensor(mask, dtype=torch.int64, device=device).expand(batch, -1)
        self.depth = torch.tensor(DEPTH, dtype=torch.int32, device=device)

    def slots(self, at):
        """Slots of token indices at [batch][n]."""
        at = at.long()
        return (self.blocks.long().gather(1, at // BLOCK) * BLOCK + at % BLOCK).reshape(-1)

    def prompt(self, tokens):
        """Writes tokens [batch][n] behind what the cache holds, their keys rotated."""
        n = tokens.shape[1]
        at = self.lens[:, None] + torch.arange(n, dtype=torch.int32, device=tokens.device)
        _, k, v = self.layer.project(tokens.reshape(-1))
        lynx.cache_append(self.geo, k, v, self.slots(at), self.K, self.V, rotary=lynx.Rotary(at.reshape(-1), self.table))
        self.lens += n

    def nodes(self, tokens, anchor_only):
        """Logits [batch][n][vocab] of the tree's first n nodes, and their keys and values."""
        n = tokens.shape[1]
        flat = tokens.reshape(-1)
        q, k, v = self.layer.project(flat)
        positions = self.lens[:, None] + self.depth[:n]
        q, k = lynx.rotary(q, k, lynx.Rotary(positions.reshape(-1), self.table))
        q, k, v = (x.unflatten(0, (self.batch, n)) for x in (q, k, v))
        o = lynx.tree_attention(self.geo, q, self.K, self.V, self.blocks, self.lens, k, v, self.mask[:, :n].contiguous(), self.workspace,
                                anchor_only=anchor_only)
        return self.layer.logits(flat, o.flatten(0, 1).flatten(1)).view(self.batch, n, -1), k, v

    def step(self, last):
        """One drafted tree from the last tokens [batch], which the cache does not hold yet.  -> the tokens that follow in each sequence (the
        accepted drafts and the one after them), and their logits."""
        tokens = last[:, None]
        for end, level in zip(self.ends, LEVELS[1:]):       # draft: a level's parents lie in the level before
            guess = self.nodes(tokens, anchor_only=True)[0]
            rank = [level[:i].count(p) for i, p in enumerate(level)]
            best = guess.topk(max(rank) + 1, -1).indices
            tokens = torch.cat((tokens, torch.stack([best[:, p, r] for p, r in zip(level, rank)], 1)), 1)
        full, k, v = self.nodes(tokens, anchor_only=False)  # verify
        chosen, drafted = full.argmax(-1).tolist(), tokens.tolist()
        paths, found = [], []
        for b in range(self.batch):
            path = [0]
            while True:
                child = [j for j, p in enumerate(PARENTS) if p == path[-1] and drafted[b][j] == chosen[b][path[-1]]]
                if not child:
                    break
                path.append(child[0])
            paths.append(path)
            found.append(([chosen[b][j] for j in path], full[b, path]))
        rows = torch.tensor([b * len(PARENTS) + j for b, path in enumerate(paths) for j in path], dtype=torch.int32, device=k.device)
        at = [(b, j) for b, path in enumerate(paths) for j in range(len(path))]
        seq = torch.tensor([b for b, _ in at], device=k.device)
        token = self.lens[seq].long() + torch.tensor([j for _, j in at], device=k.device)
        slots = self.blocks[seq, token // BLOCK].long() * BLOCK + token % BLOCK
        lynx.cache_append(self.geo, k.flatten(0, 1), v.flatten(0, 1), slots, self.K, self.V, rows=rows)   # (rotated already)
        self.lens += torch.tensor([len(path) for path in paths], dtype=torch.int32, device=k.device)
        return found

    def pages(self):
        """What the cache holds: keys and values BF16 [tokens][kv_heads][128], sequence by sequence."""
        offsets = torch.cat((self.lens.new_zeros(1), self.lens.cumsum(0, dtype=torch.int32)))
        return lynx.cache_read(self.geo, self.K, self.V, self.blocks, None, offsets, int(offsets[-1]))


def decode(layer, prompt, n_tokens):
    """Decodes at least n_tokens behind a prompt [batch][n].  -> decoder, each sequence's tokens and their logits, steps."""
    d = Decoder(layer, len(prompt), prompt.shape[1] + n_tokens + 2 * len(LEVELS))
    if prompt.shape[1] > 1:
        d.prompt(prompt[:, :-1])
    last, got, steps = prompt[:, -1], [([], []) for _ in prompt], 0
    while min(len(t) for t, _ in got) < n_tokens:
        active = [len(t) < n_tokens for t, _ in got]
        before = d.lens.clone()
        found = d.step(last)
        for b, (tokens, logits) in enumerate(found):
            if active[b]:
                got[b][0].extend(tokens)
                got[b][1].extend(logits)
        # (a sequence that is done stays where it is: what was written behind its end is never read)
        keep = torch.tensor(active, device=last.device)
        d.lens = torch.where(keep, d.lens, before)
        last = torch.tensor([t[-1] for t, _ in got], device=last.device)
        steps += 1
    return d, [t for t, _ in got], [x for _, x in got], steps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--context", type=int, default=4096)
    a = ap.parse_args()
    layer = Layer()
    prompt = torch.randint(layer.vocab, (a.batch, a.context), generator=torch.Generator().manual_seed(1)).cuda()
    decode(layer, prompt, 4)     # (warm up)
    torch.cuda.synchronize()
    t = time.perf_counter()
    d, tokens, _, steps = decode(layer, prompt, a.tokens)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    total = sum(map(len, tokens))
    k, _ = d.pages()
    print(f"{a.batch} sequences, context {a.context}: {total} tokens in {steps} steps ({total / steps / a.batch:.2f} a step and sequence), "
          f"{t * 1e3 / steps:.2f} ms a step; the cache holds {len(k)} tokens")


if __name__ == "__main__":
    main()
