"""The serving example's limits: what does not fit into a place's table is refused before any block is taken; what just fits is served."""
import pytest
import torch

import test_gpu_latent_serving as serving

pytestmark = pytest.mark.gpu
example = serving.example


def _server(capacity, blocks=12):
    return example.Server(example.Layer(vocab=64, dim=128, heads=4), 2, blocks, capacity)


def _prompt(n):
    return torch.randint(64, (n,), generator=torch.Generator().manual_seed(n)).cuda()


@pytest.mark.parametrize("n", [0, 97, 98, 130, 1000])
def test_a_prompt_that_does_not_fit_takes_no_blocks(n):
    server = _server(96)
    assert server.start(1, _prompt(40))
    before = [x.clone() for x in (server.pool.ring, server.pool.state, server.table, server.lens)]
    for _ in range(2):
        with pytest.raises(ValueError):
            server.start(0, _prompt(n))
    assert all(torch.equal(x, y) for x, y in zip(before, (server.pool.ring, server.pool.state, server.table, server.lens)))
    assert server.start(0, _prompt(96))


def test_a_request_that_would_outgrow_its_place_is_refused():
    server = _server(96)
    with pytest.raises(ValueError):
        example.serve(server, [_prompt(10), _prompt(60)], 38)
    assert int(server.pool.state[1]) == 12 and not server.lens.any()
    got, _ = example.serve(server, [_prompt(10), _prompt(60)], 37)     # 59 + 37 tokens
    assert [len(x) for x in got] == [37, 37] and int(server.pool.state[1]) == 12


def test_positions_up_to_the_end_of_the_last_block_have_angles():
    """A capacity that is no multiple of a block."""
    server = _server(70)
    assert server.capacity == 96 and len(server.angles) == 96
    got, _ = example.serve(server, [_prompt(60)], 37)
    assert len(got[0]) == 37
