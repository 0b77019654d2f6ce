"""The bookkeeping of the serving example without a GPU: the definition hands out the blocks, the layers compute nothing."""
import copy

import numpy as np
import pytest
import torch

import attn_oracle
from paper_2411_19379_amd import prefix_cache as pc
from test_gpu_attention_example import _example


class NoLayers:
    """What the server asks of its model."""

    qkv = [None]
    embedding = torch.zeros(1000, 8)

    def caches(self, n_blocks, block_size):
        return []

    def forward(self, tokens, step, cu, cached, caches, max_new=0):
        return torch.zeros(len(tokens), 8)


def _assign(attn):
    def assign_blocks(block_size, total_tokens, cu, cached, table, free, n_free, shared_tail=None, in_place=False):
        assert in_place and total_tokens == int(cu[-1])
        shared = None if shared_tail is None else shared_tail.numpy()
        got = attn_oracle.assign(block_size, cu.numpy(), cached.numpy(), table.numpy(), free.numpy(), int(n_free), shared)
        got = [torch.from_numpy(np.ascontiguousarray(g)) for g in got]
        table.copy_(got[0])
        return attn.Step(table, *got[1:])
    return assign_blocks


@pytest.fixture
def server(monkeypatch):
    example = _example()
    monkeypatch.setattr(example.attn, "assign_blocks", _assign(example.attn))
    return example.Server(NoLayers(), n_blocks=8, block_size=4, most_tokens=60, capacity_bytes=1 << 20)


def _state(server):
    return copy.deepcopy((server.free, server.holders, server.sequences))


FIRST = (list(range(10)), [500, 501, 502])  # 13 tokens, 4 blocks
MORE = FIRST[0] + FIRST[1]                  # resumes inside the fourth


@pytest.mark.parametrize("requests", [
    # the prefill lacks blocks, neither token behind it needs one
    [(MORE + list(range(100, 121)), [7, 8])],
    [(list(range(200, 202)), [1, 2]), (MORE + list(range(100, 120)), [7, 8])],
    # a token in the middle does, the last one not
    [(MORE + list(range(100, 116)), [1, 2, 3, 4, 5, 6])]])
def test_blocks_missing_in_any_step_are_noticed(server, requests):
    """Rows computed without keys of their own are not returned, nothing is held, and the hits' pins are given back."""
    server.serve([FIRST])
    before = _state(server)
    with pytest.raises(RuntimeError, match="missing"):
        server.serve(requests)
    assert _state(server) == before
    look = server.cache.begin(requests[-1][0], server.now)
    assert look.hit_len == len(MORE)
    server.cache.abort(requests[-1][0], look)
    with pytest.raises(pc.PrefixCacheError):
        server.cache.abort(requests[-1][0], look)  # no pin is left
    lens, rows = server.serve([(MORE + [3, 4], [9])])  # the server goes on
    assert lens == [len(MORE)] and rows[0].shape[0] == 3
    assert -1 not in server.free and all(b >= 0 for s in server.sequences.values() for b in s)


def test_a_step_that_fails_gives_back_the_pins(server, monkeypatch):
    server.serve([FIRST])
    before = _state(server)
    with monkeypatch.context() as m:
        m.setattr(NoLayers, "forward", lambda *a, **k: 1 / 0)
        with pytest.raises(ZeroDivisionError):
            server.serve([(MORE + [1], [2])])
    assert _state(server) == before
    look = server.cache.begin(MORE + [1], server.now)
    server.cache.abort(MORE + [1], look)
    with pytest.raises(pc.PrefixCacheError):
        server.cache.abort(MORE + [1], look)
