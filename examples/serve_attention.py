"""Multi-turn serving of a model's attention layers behind the prefix cache, on one MI355X.

    python examples/serve_attention.py [--sessions 24] [--batch 8] [--window 0] [--dtype bf16]

Requests of a synthetic chat trace (the shape of Section 5.1's workloads) are served in batches.  For each one the prefix cache
names the cached sequence to resume from (Section 4.1); its blocks go into the request's row of the block table, and the new
tokens of the whole batch run as one packed prefill, then token by token:

    assign_blocks   once per step: blocks, slots and positions of the new tokens; a hit that ends inside a block of the cached
                    sequence gets a block of its own in its place
    rope_append     once per layer: rotary positions, k and v into the cache, the copy of that block
    attend          once per layer: attention over everything in the cache

The lengths stay on the GPU; the host keeps the free list and counts how many cached sequences hold a block.  The rest of the
layer (norms, projections) is plain torch, and the outputs are the trace's, fed back one by one as sampled tokens would be.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_19379_amd import attention as attn  # noqa: E402
from paper_2411_19379_amd import prefix_cache as pc  # noqa: E402
from workloads.traces import make_trace  # noqa: E402


class Layers:
    """A stack of attention layers with random weights."""

    def __init__(self, n_layers, d_model, n_q_heads, n_kv_heads, head_dim, vocab, dtype, max_positions, window=0, sinks=0,
                 device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)
        make = lambda *s: (torch.randn(s, generator=g) / s[-1] ** 0.5).to(dtype).to(device)
        self.hq, self.hkv, self.d = n_q_heads, n_kv_heads, head_dim
        self.window, self.sinks = window, sinks
        self.embedding = torch.randn((vocab, d_model), generator=g).to(dtype).to(device)
        self.qkv = [make((n_q_heads + 2 * n_kv_heads) * head_dim, d_model) for _ in range(n_layers)]
        self.out = [make(d_model, n_q_heads * head_dim) for _ in range(n_layers)]
        self.rotary = attn.rotary_table(max_positions, head_dim, device=device)

    def caches(self, n_blocks, block_size):
        like = dict(dtype=self.embedding.dtype, device=self.embedding.device)
        return [[torch.empty((n_blocks, self.hkv, block_size, self.d), **like) for _ in "kv"] for _ in self.qkv]

    def forward(self, tokens, step, cu, cached, caches, max_new=0):
        x = self.embedding[tokens]
        for w_qkv, w_out, (k_cache, v_cache) in zip(self.qkv, self.out, caches):
            h = torch.nn.functional.rms_norm(x, x.shape[-1:])
            # q, k and v are parts of the projection's rows; nothing is copied to take them apart
            q, k, v = (h @ w_qkv.T).view(-1, self.hq + 2 * self.hkv, self.d).split((self.hq, self.hkv, self.hkv), 1)
            q = attn.rope_append(q, k, v, step.positions, step.slots, self.rotary, k_cache, v_cache, copies=step.copies)
            y = attn.attend(q, k_cache, v_cache, step.table, cu, cached, window=self.window, sinks=self.sinks, max_new=max_new)
            x = x + y.flatten(1) @ w_out.T
        return x


class Server:
    def __init__(self, model: Layers, n_blocks: int, block_size: int, most_tokens: int, capacity_bytes: int):
        self.model, self.block_size, self.width = model, block_size, -(-most_tokens // block_size)
        self.device = model.embedding.device
        self.caches = model.caches(n_blocks, block_size)
        self.free = list(range(n_blocks))
        self.holders = [0] * n_blocks       # cached sequences that hold a block
        self.sequences = {}                 # handle -> blocks of a cached sequence
        self.cache = pc.PrefixCache(n_attn=len(model.qkv), n_ssm=1, n_mlp=1, d_model=model.embedding.shape[1], d_state=16,
                                    capacity_bytes=capacity_bytes, alpha=1.0)
        self.now = self.next_handle = 0

    def _ints(self, values):
        return torch.tensor(values, dtype=torch.int32).to(self.device)

    def _hold(self, blocks):
        self.next_handle += 1
        self.sequences[self.next_handle] = blocks
        for b in blocks:
            self.holders[b] += 1
        return self.next_handle

    def _release(self, handle):
        for b in self.sequences.pop(handle):
            self.holders[b] -= 1
            if self.holders[b] == 0:
                self.free.append(b)

    def _step(self, tokens, new, cached, table, pool, n_free, shared_tail=None):
        """One forward pass of new[b] tokens of every sequence; returns its step and the last layer's rows."""
        cu = torch.zeros(len(new) + 1, dtype=torch.int32)
        cu[1:] = torch.tensor(new).cumsum(0)
        cu = cu.to(self.device)
        step = attn.assign_blocks(self.block_size, len(tokens), cu, cached, table, pool, n_free, shared_tail=shared_tail, in_place=True)
        return step, self.model.forward(torch.tensor(tokens).to(self.device), step, cu, cached, self.caches, max_new=max(new))

    def serve(self, requests):
        """Serves (input, output) pairs as one batch.  Returns per request the tokens that were not computed and the rows of
        the last layer for all that were."""
        self.now += 1
        looks = []
        try:
            for inp, _ in requests:
                looks.append(self.cache.begin(inp, self.now))
            lens, results, table, left = self._compute(requests, looks)
        except BaseException:  # nothing is held yet: the hits' pins go back, the free list is as it was
            for (inp, _), look in zip(requests, looks):
                self.cache.abort(inp, look)
            raise
        del self.free[left:]
        for (inp, out), look, row in zip(requests, looks, table):
            full = inp + out
            branch = self._hold(row[:-(-look.checkpoint_pos // self.block_size)]) if look.checkpoint_pos else None
            final = self._hold(row[:-(-len(full) // self.block_size)])
            evicted, rejected = self.cache.finish(full, look, branch, final, self.now)
            for handle in evicted + rejected:
                self._release(handle)
        return lens, results

    def _compute(self, requests, looks):
        """The prefill and the tokens behind it.  Returns per request the tokens that were not computed and the rows of the others,
        the table, and how many blocks are left of the free list."""
        table = torch.full((len(requests), self.width), -1, dtype=torch.int32)
        for b, look in enumerate(looks):
            if look.hit_len:
                blocks = self.sequences[look.hit_handle][:-(-look.hit_len // self.block_size)]
                table[b, :len(blocks)] = torch.tensor(blocks, dtype=torch.int32)
        table, pool = table.to(self.device), self._ints(self.free)
        lens = [look.hit_len for look in looks]
        cached = self._ints(lens)
        new = [len(inp) - n for (inp, _), n in zip(requests, lens)]
        tokens = [t for (inp, _), n in zip(requests, lens) for t in inp[n:]]
        # a hit's last block may be read by other requests and be written to by the one that it belongs to
        step, rows = self._step(tokens, new, cached, table, pool, self._ints([len(self.free)]), self._ints([int(n > 0) for n in lens]))
        results = [[r] for r in rows.split(new)]
        missing = step.counts[1:]  # of every step: a later one may need none
        for i in range(max(len(out) for _, out in requests)):
            cached = cached + self._ints(new)
            new = [int(i < len(out)) for _, out in requests]
            step, rows = self._step([out[i] for _, out in requests if i < len(out)], new, cached, table, pool, step.counts[:1])
            missing = missing + step.counts[1:]
            for b, r in zip([b for b, n in enumerate(new) if n], rows.split(1)):
                results[b].append(r)
        left, missing = torch.cat([step.counts[:1], missing]).tolist()
        if missing:
            raise RuntimeError(f"{missing} blocks missing: the cache's capacity leaves too few for a batch")
        return lens, [torch.cat(r) for r in results], table.tolist(), left


def run(sessions=24, batch=8, window=0, sinks=0, dtype="bf16", n_layers=4, d_model=1024, n_q_heads=16, n_kv_heads=4, head_dim=64,
        block_size=16, n_blocks=8192, prompt_len=(200, 600), user_len=(10, 120), out_len=(5, 40), capacity_bytes=1 << 28, seed=0,
        on_batch=None):
    """Serves a trace; returns what it took.  `on_batch(server, requests, skipped, rows)` sees every batch."""
    types = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    trace = make_trace(seed, n_sessions=sessions, prompt_len=prompt_len, user_len=user_len, out_len=out_len)
    most = max(len(i) + len(o) for i, o in trace)
    model = Layers(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, 1000, types[dtype], most, window, sinks, seed=seed)
    server = Server(model, n_blocks, block_size, most, capacity_bytes)
    tokens = skipped = steps = 0
    torch.cuda.synchronize()
    start = time.time()
    for at in range(0, len(trace), batch):
        requests = trace[at:at + batch]
        lens, rows = server.serve(requests)
        skipped += sum(lens)
        tokens += sum(len(i) + len(o) for i, o in requests)
        steps += 1 + max(len(o) for _, o in requests)
        if on_batch:
            on_batch(server, requests, lens, rows)
    torch.cuda.synchronize()
    return dict(requests=len(trace), tokens=tokens, skipped=skipped, steps=steps, seconds=time.time() - start,
                blocks_free=len(server.free), blocks_held=sum(h > 0 for h in server.holders), blocks=n_blocks)


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--sessions", type=int, default=24)
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--window", type=int, default=0, help="tokens that a layer looks back, 0: all")
    p.add_argument("--sinks", type=int, default=0, help="first tokens that stay visible in front of the window")
    p.add_argument("--dtype", choices=["bf16", "f16", "f32"], default="bf16")
    r = run(**vars(p.parse_args()))
    print(f"{r['requests']} requests, {r['tokens']} tokens, {r['skipped']} of them not computed again ({100 * r['skipped'] / r['tokens']:.1f} %), "
          f"{r['steps']} steps in {r['seconds']:.2f} s, {r['blocks_held']} of {r['blocks']} blocks held")
