"""Serving requests that come and go over one pool of quantised latents: how the entry points around a cache of latents work together.

    python examples/latent_serving.py [--tokens 64] [--batch 8] [--context 4096]

One attention layer with random weights stands for a model whose keys and values are expanded from one latent a token.  Each request has a place in
the batch; a prompt is written 64 positions at a time, a decode step is one captured graph for all places, whichever of them are in use:

    plan_blocks       blocks for what requests grow by, slots and positions of their new tokens; blocks of requests that end go back
    norm_rotary       the rotary parts of the queries, turned
    latent_append     the tokens' latents, normed and quantised, and their rotary keys, turned
    latent_attention  all heads over the latents, absorbed form
    latent_read       what the cache holds, as BF16, for an engine that wants the expanded form
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_01831_b200 as lynx  # noqa: E402

BLOCK, CHUNK = 32, 64
LATENT, ROPE, HEAD = 512, 64, 128


class Layer:
    """An embedding, one attention layer in absorbed form, and the embedding again for the next token."""

    def __init__(self, vocab=1024, dim=512, heads=16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device=device) / shape[-2] ** 0.5).to(torch.bfloat16)

        self.heads, self.vocab = heads, vocab
        self.embed = torch.randn(vocab, dim, generator=g, device=device).to(torch.bfloat16)
        self.down = weight(dim, LATENT + ROPE)
        self.norm = (1.0 + 0.1 * torch.randn(LATENT, generator=g, device=device)).to(torch.bfloat16)
        self.query, self.query_rope = weight(dim, heads * HEAD), weight(dim, heads * ROPE)
        self.key_up, self.value_up = weight(heads, HEAD, LATENT), weight(heads, LATENT, HEAD)   # (a key is latent times key_up^T)
        self.out = weight(heads * HEAD, dim)

    def latents(self, tokens):
        """Latents [T][512] and rotary keys [T][64] of tokens: views of one product."""
        return (self.embed[tokens] @ self.down).split((LATENT, ROPE), 1)

    def queries(self, tokens, rotary):
        """Absorbed queries [T][heads][512] and their rotary part [T][heads][64], turned."""
        x = self.embed[tokens]
        q = torch.einsum("thd,hdc->thc", (x @ self.query).view(-1, self.heads, HEAD), self.key_up).contiguous()   # (the product is head by head)
        qr = (x @ self.query_rope).view(-1, self.heads, ROPE)
        return q, lynx.norm_rotary(qr, None, None, rotary, q_out=qr)[0]

    def next(self, tokens, o):
        """The tokens that follow, from attention's output [T][heads][512]."""
        v = torch.einsum("thc,hcd->thd", o, self.value_up).flatten(1)
        return ((self.embed[tokens] + v @ self.out) @ self.embed.t()).argmax(-1)


class Server:
    def __init__(self, layer, batch, blocks, capacity):
        device = layer.embed.device
        self.layer, self.batch = layer, batch
        self.geo = lynx.Geometry(layer.heads, 4, BLOCK, blocks, -(-capacity // BLOCK))
        self.planes = lynx.Planes(torch.zeros(blocks, 4, BLOCK, 64, dtype=torch.uint8, device=device),
                                  torch.zeros(blocks, 4, BLOCK, 64, dtype=torch.uint8, device=device), torch.zeros(blocks, 4, BLOCK, 2, device=device))
        self.pages = torch.zeros(blocks, BLOCK, ROPE, dtype=torch.bfloat16, device=device)
        self.pool = lynx.make_block_pool(blocks, device)
        self.table = torch.zeros(batch, self.geo.max_blocks_per_seq, dtype=torch.int32, device=device)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=device)
        self.active = torch.zeros(batch, dtype=torch.int32, device=device)     # 1: the place decodes
        self.last = torch.zeros(batch, dtype=torch.int64, device=device)       # its last token, not in the cache yet
        self.capacity = self.geo.max_blocks_per_seq * BLOCK                    # tokens of a place's table: plan_blocks clamps lengths to it
        self.angles = lynx.rotary_table(self.capacity, ROPE // 2, device=device)
        self.ws_step = lynx.make_latent_workspace(self.geo, batch, 1, device)
        self.ws_chunk = lynx.make_latent_workspace(self.geo, 1, CHUNK, device)
        self.graph = None

    def plan(self, new_lens, max_tokens):
        plan = lynx.plan_blocks(self.geo, self.pool, self.table, self.lens, new_lens, max_tokens)
        self.lens.copy_(plan.lens)
        return plan

    def write(self, tokens, slots, rotary, rows=None):
        c, k = self.layer.latents(tokens)
        lynx.latent_append(self.geo, c, k, slots, self.planes, self.pages, self.layer.norm, rows=rows, rotary=rotary)

    def start(self, at, prompt):
        """Puts a request with prompt [n] into the free place `at`, 64 positions at a time.  False: there are no blocks for it, and nothing has changed."""
        n = len(prompt)
        if not 1 <= n <= self.capacity:     # (its last token is not in the cache yet, but will be)
            raise ValueError(f"a prompt must have 1 to {self.capacity} tokens")
        plan = lynx.plan_blocks(self.geo, self.pool, self.table, self.lens, self.grown(at, n - 1), n - 1)
        if int(plan.lens[at]) < n - 1:      # (a request that does not get its blocks stays as it is)
            return False
        for i in range(0, n - 1, CHUNK):
            part = prompt[i:min(i + CHUNK, n - 1)]
            rotary = lynx.Rotary(plan.positions[i:i + len(part)], self.angles)
            self.write(part, plan.slots[i:i + len(part)], rotary)
            q, qr = self.layer.queries(part, rotary)
            self.attend(q[None], qr[None], self.table[at:at + 1], self.lens.new_full((1,), i + len(part)), self.ws_chunk)   # (a deeper model's next layer takes it)
        self.lens.copy_(plan.lens)
        self.last[at] = prompt[-1]
        self.active[at] = 1
        return True

    def grown(self, at, n):
        lens = self.lens.clone()
        lens[at] = n
        return lens

    def end(self, at):
        """Ends the request: its blocks go back to the pool."""
        self.plan(self.grown(at, 0), 0)
        self.active[at] = 0

    def attend(self, q, qr, table, lens, ws):
        return lynx.latent_attention(self.geo, q, qr, self.planes, self.pages, table, lens, ws)

    def step_once(self):
        before = self.lens.clone()
        plan = self.plan(self.lens + self.active, self.batch)
        grew = self.lens > before
        # the row of each place's new token; places without one have none, and write nothing
        row = plan.offsets[:-1].clamp(max=self.batch - 1).long()
        slots = torch.where(grew, plan.slots[row], -1)
        rotary = lynx.Rotary(before, self.angles)
        self.write(self.last, slots, rotary)
        q, qr = self.layer.queries(self.last, rotary)
        o = self.attend(q[:, None], qr[:, None], self.table, torch.where(grew, self.lens, 0), self.ws_step)
        self.last.copy_(torch.where(grew, self.layer.next(self.last, o[:, 0]), self.last))

    def step(self):
        """One token for every place in use."""
        if self.graph is None:
            keep = [x.clone() for x in (self.lens, self.last, self.pool.ring, self.pool.state, self.table)]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                self.step_once()                # (once outside of the graph, for what is set up on first use)
            torch.cuda.current_stream().wait_stream(side)
            for x, y in zip((self.lens, self.last, self.pool.ring, self.pool.state, self.table), keep):
                x.copy_(y)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.step_once()
        self.graph.replay()

    def held(self):
        """What the cache holds: latents BF16 [tokens][512] and rotary keys [tokens][64], place by place."""
        offsets = torch.cat((self.lens.new_zeros(1), self.lens.cumsum(0, dtype=torch.int32)))
        return lynx.latent_read(self.geo, self.planes, self.pages, self.table, None, offsets, int(offsets[-1]))


def serve(server, prompts, n_tokens):
    """Serves all prompts, n_tokens each, as many at a time as there are places and blocks.  -> each prompt's tokens, decode steps."""
    if any(len(x) - 1 + n_tokens > server.capacity for x in prompts):      # (a place that is full gets no further token)
        raise ValueError(f"a request must end within {server.capacity} tokens")
    waiting, place, got, steps = list(range(len(prompts))), [None] * server.batch, [[] for _ in prompts], 0
    while waiting or any(r is not None for r in place):
        for at in range(server.batch):
            if place[at] is None and waiting and server.start(at, prompts[waiting[0]]):
                place[at] = waiting.pop(0)
        if not any(r is not None for r in place):
            raise RuntimeError("a prompt is longer than the pool")
        before = server.lens.tolist()
        server.step()
        steps += 1
        after, tokens = server.lens.tolist(), server.last.tolist()
        if after == before:
            raise RuntimeError("no request can go on: the pool is too small for them")
        for at, r in enumerate(place):
            if r is None:
                continue
            if after[at] > before[at]:          # (one without a block waits until others end)
                got[r].append(tokens[at])
            if len(got[r]) == n_tokens:
                server.end(at)
                place[at] = None
    return got, steps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--context", type=int, default=4096)
    a = ap.parse_args()
    layer = Layer()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(layer.vocab, (a.context // 2 + a.context * i // (4 * a.batch),), generator=g).cuda() for i in range(2 * a.batch)]
    capacity = a.context + a.tokens
    server = Server(layer, a.batch, a.batch * (-(-capacity // BLOCK)), capacity)
    serve(server, prompts[:1], 4)     # (warm up)
    torch.cuda.synchronize()
    t = time.perf_counter()
    got, steps = serve(server, prompts, a.tokens)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"{len(prompts)} requests in {a.batch} places: {sum(map(len, got))} tokens in {steps} steps, {t:.2f} s with their prompts; "
          f"{int(server.pool.state[1])} of {server.geo.num_blocks} blocks are free again")


if __name__ == "__main__":
    main()
