"""The serving example on the GPU: every row of every request against the same layers in 64 bits over the whole sequence."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_attention", os.path.join(ROOT, "examples", "serve_attention.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _rows64(model, tokens):
    x = model.embedding[torch.tensor(tokens, device=model.embedding.device)].double()
    n, g = len(tokens), model.hq // model.hkv
    pos = torch.arange(n, device=x.device)
    seen = pos[None] <= pos[:, None]
    if model.window:
        seen &= (pos[:, None] - pos[None] < model.window) | (pos[None] < model.sinks)
    cos, sin = model.rotary[:n, :1].double(), model.rotary[:n, 1:].double()
    turn = lambda a, b: torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    for w_qkv, w_out in zip(model.qkv, model.out):
        h = x / (x.square().mean(-1, keepdim=True) + torch.finfo(torch.float32).eps).sqrt()
        q, k, v = (h @ w_qkv.double().T).view(n, -1, model.d).split((model.hq, model.hkv, model.hkv), 1)
        q, k = turn(*q.chunk(2, -1)), turn(*k.chunk(2, -1))
        y = torch.empty_like(q)
        for i in range(model.hq):
            s = (q[:, i] @ k[:, i // g].T) * model.d ** -0.5
            y[:, i] = torch.softmax(s.masked_fill(~seen, -float("inf")), 1) @ v[:, i // g]
        x = x + y.flatten(1) @ w_out.double().T
    return x


@pytest.mark.parametrize("window,sinks,block_size,capacity", [(0, 0, 16, 1 << 28), (0, 0, 16, 1 << 20), (40, 4, 8, 1 << 28)])
def test_serving_matches_the_whole_sequences(window, sinks, block_size, capacity):
    """In fp32: a layer is five sums of at most 256 products and a softmax whose scores are some tens, each off by less than
    256 * 2^-24 = 1.5e-5 of its size, so two layers stay below 1e-3 of the largest value; one wrong key, position or block
    moves rows by tenths."""
    seen = dict(hits=0)

    def check(server, requests, skipped, rows):
        for (inp, out), n, got in zip(requests, skipped, rows):
            want = _rows64(server.model, inp + out)[n:]
            assert got.shape == want.shape
            off = float((got.double() - want).abs().max() / want.abs().max())
            assert off <= 1e-3, (off, n, len(inp), len(out))
            seen["hits"] += n > 0
        held = {b for blocks in server.sequences.values() for b in blocks}
        assert held.isdisjoint(server.free) and len(held) + len(server.free) == len(server.holders)

    r = _example().run(sessions=10, batch=5, window=window, sinks=sinks, dtype="f32", n_layers=2, d_model=256, n_q_heads=4, n_kv_heads=2,
                       block_size=block_size, n_blocks=1500, prompt_len=(40, 150), user_len=(1, 60), out_len=(1, 30),
                       capacity_bytes=capacity, on_batch=check)
    print(r, flush=True)
    assert seen["hits"] >= 5 and r["skipped"] > 0
