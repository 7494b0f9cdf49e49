"""The example that serves requests over a pool of latents: what it attends to against 64 bits, what its cache holds against plain torch, and that
no block is lost, in a pool that is too small for all requests at once."""
import importlib.util
import os

import pytest
import torch

import paper_2607_01831_b200 as lynx

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


def _load(path):
    spec = importlib.util.spec_from_file_location(os.path.basename(path)[:-3], path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


example = _load(os.path.join(os.path.dirname(HERE), "examples", "latent_serving.py"))
bounds = _load(os.path.join(HERE, "test_gpu_latent_attention.py"))


class _Held(bounds.Cache):
    """A server's cache as the attention's test reads one."""

    def __init__(self, server, table, lens):
        self.lens, self.bt, self.table = lens.tolist(), example.BLOCK, table.cpu()
        self.planes, self.pages = server.planes, server.pages


class _Watched(example.Server):
    """Keeps what its last attention read and wrote: of a captured step, the graph's own tensors."""

    def attend(self, q, qr, table, lens, ws):
        out = super().attend(q, qr, table, lens, ws)
        self.seen = (q, qr, table, lens, out)
        if self.graph is None and not torch.cuda.is_current_stream_capturing():
            self.check()
        return out

    def check(self):
        q, qr, table, lens, out = self.seen
        bounds._check(_Held(self, table, lens), q, qr, out, None, True, False)


def _plain(layer, tokens, angles):
    """Latents and rotary keys as the cache is to hold them, in 64 bits: [T][512] and [T][64]."""
    c, k = (x.double() for x in layer.latents(tokens))
    c = c / (c.square().mean(1, keepdim=True) + 1e-6).sqrt() * layer.norm.double()
    cos, sin = angles[:len(tokens)].double().split(32, 1)
    return c, torch.cat((k[:, :32] * cos - k[:, 32:] * sin, k[:, 32:] * cos + k[:, :32] * sin), 1)


@pytest.mark.parametrize("captured", [True, False])
def test_requests_come_and_go(captured):
    layer = example.Layer(vocab=256, dim=256, heads=8)
    # 26 blocks of 32 tokens: 3 places, of requests that end with 3 to 13 blocks
    server = _Watched(layer, 3, 26, 448)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(256, (n,), generator=g).cuda() for n in (90, 1, 300, 64, 395, 33, 2)]
    history = {}     # prompts by place

    real_start, real_step = server.start, server.step if captured else server.step_once

    def start(at, prompt):
        ok = real_start(at, prompt)
        if ok:
            history[at] = prompt.tolist()
        return ok

    def step():
        before = server.lens.tolist()
        real_step()
        server.check()
        assert int(server.pool.state[1]) == 26 - sum(-(-n // 32) for n in server.lens.tolist())
        # what each place holds are the latents of its prompt and its tokens but the last
        c, k = server.held()
        row = 0
        for at, n in enumerate(server.lens.tolist()):
            if n == 0:
                continue
            tokens = torch.tensor(history[at][:n]).cuda()
            assert len(tokens) == n
            want_c, want_k = _plain(layer, tokens, server.angles)
            # BF16's rounding of what is read back, half a quantisation step of 128 channels, and the projection's own rounding, which may go the other way in
            # a product of another size: a step, 2^-7, of a value, and of the norm's mean at most as much again
            rows = want_c.view(n, 4, 128)
            span, most = rows.amax(2) - rows.amin(2), rows.abs().amax(2)
            bound = (span * (1 + 2.0 ** -6) / 510 + (2.0 ** -8 + 2.0 ** -6) * most)[..., None].expand(-1, -1, 128).flatten(1)
            assert ((c[row:row + n].double() - want_c).abs() <= bound).all()
            pair = (want_k[:, :32].square() + want_k[:, 32:].square()).sqrt().repeat(1, 2)      # (as long as before it was turned)
            assert ((k[row:row + n].double() - want_k).abs() <= (2.0 ** -8 + 2.0 ** -7 * 2 ** 0.5) * pair + 1e-12).all()
            row += n
        assert row == len(c)
        last, after = server.last.tolist(), server.lens.tolist()
        for at in history:
            if after[at] > before[at]:
                history[at].append(last[at])

    server.start, server.step = start, step
    got, steps = example.serve(server, prompts, 20)
    assert all(len(x) == 20 for x in got) and steps >= 3 * 20
    assert int(server.pool.state[1]) == 26 and sorted(server.pool.ring.tolist()) == list(range(26)) and not server.lens.any()
    lynx.check(server.ws_step)
    lynx.check(server.ws_chunk)
