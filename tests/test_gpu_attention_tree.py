"""Steps that check trees of drafted tokens, on the GPU: each operator against its definition in 64 bits, a run of them as a server
makes it against decoding token by token, captured into a graph, on another stream."""
from __future__ import annotations

import random

import numpy as np
import pytest
import torch

import attn_helpers as ah
import tree_helpers as th
import tree_oracle
from paper_2411_19379_amd import attention as attn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(v, dtype=torch.int32):
    return torch.as_tensor(np.asarray(v), dtype=dtype, device=DEV)


def _attend(p, **more):
    args = (p.q.to(DEV), p.k_cache.to(DEV), p.v_cache.to(DEV), _ints(p.table), _ints(p.cu), _ints(p.cached), _ints(p.positions), _ints(p.bits))
    out, lse = attn.attend_tree(*args, scale=p.scale, window=p.window, sinks=p.sinks, max_new=p.max_new, return_lse=True, **more)
    return out.cpu().double().numpy(), lse.cpu().numpy()


@pytest.mark.parametrize("new,cached,words,window,sinks", [([1], [0], 1, 0, 0), ([17, 0, 33, 2], [5, 0, 100, 31], 2, 0, 0),
                                                          ([70, 300], [3, 40], 10, 4, 0), ([64, 40], [0, 9], 2, 3, 12), ([1024], [7], 32, 0, 0)])
def test_draft_tree(new, cached, words, window, sinks):
    rng = random.Random(sum(new))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    parents = np.array([x for n in new for x in tree_oracle.random_parents(rng, n, 0.9, 0.05)] + [0, 1, 2], np.int32)
    positions, seen = tree_oracle.draft_tree(parents, cu, cached, words, window, sinks)
    tree = attn.draft_tree(_ints(parents), _ints(cu), _ints(cached), 32 * words, window=window, sinks=sinks)
    assert np.array_equal(tree.positions.cpu(), positions)
    assert np.array_equal(tree.seen.cpu(), tree_oracle.bits_of(seen, words))


@pytest.mark.parametrize("bits", ["tree", "any"])
@pytest.mark.parametrize("name", sorted(th.CASES))
def test_attend(name, bits):
    p = th.make(21, *th.CASES[name], bits=bits, holes=0.03)
    out, lse = _attend(p)
    ah.check(p, out, lse, name, th.reference(p))
    again = _attend(p)
    assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])


@pytest.mark.parametrize("hq,hkv,d,bs,dtype,new,cached,window", [
    (32, 8, 128, 16, "bf16", [17], [2000], 0), (8, 2, 64, 32, "f16", [64, 40, 3], [1500, 700, 0], 0), (16, 1, 128, 16, "bf16", [30, 64], [900, 333], 0),
    (5, 5, 64, 64, "bf16", [256, 100], [300, 1000], 100), (4, 4, 128, 8, "f32", [50], [1200], 0), (64, 1, 64, 16, "f16", [9], [800], 0)])
def test_attend_long(hq, hkv, d, bs, dtype, new, cached, window):
    p = th.make(5, hq, hkv, d, bs, dtype, new, cached, window, 3 if window else 0, max(new))
    out, lse = _attend(p)
    ah.check(p, out, lse, "long", th.reference(p))


def test_attend_chain_is_attend():
    """The bits of a chain: what attend computes, bit for bit where the same kernel runs on the same tiles."""
    p = th.make(3, 8, 2, 64, 16, "bf16", [40, 5, 1], [100, 31, 64], max_new=40)
    p.positions, p.seen = tree_oracle.draft_tree(np.concatenate([np.arange(n) - 1 for n in p.new]), p.cu, p.cached, p.words)
    p.bits = tree_oracle.bits_of(p.seen, p.words)
    out, lse = _attend(p)
    ref = ah.reference(p)
    ah.check(p, out, lse, "chain", ref)


@pytest.mark.parametrize("seed,batch,most,bs,more", [(1, 1, 20, 16, {}), (2, 7, 40, 8, {}), (3, 130, 30, 4, {}), (4, 5, 200, 16, dict(vocabulary=1)),
                                                    (5, 9, 130, 16, dict(holes=0.3)), (7, 1500, 4, 8, {})])
def test_accept_and_keep(seed, batch, most, bs, more):
    p = th.accept_problem(seed, batch, most, bs, **more)
    free = np.arange(5000, 5060, dtype=np.int32)
    want = tree_oracle.accept_path(p["tokens"], p["parents"], p["choices"], p["cu"], p["cached"], p["table"], bs, free, 7)
    arrays = [_ints(p[k]) for k in ("tokens", "parents", "choices", "cu", "cached")]
    free_dev = _ints(free)
    kept = attn.accept_path(*arrays, block_size=bs, table=_ints(p["table"]), free_blocks=free_dev, n_free=_ints([7]))
    for got, w in zip((*kept[:4], free_dev, kept.n_free), (*want[:5], [want[5]])):
        assert np.array_equal(got.cpu(), w)
    plain = attn.accept_path(*arrays)
    assert plain.n_free is None and all(torch.equal(a, b) for a, b in zip(plain[:4], kept[:4]))
    g = torch.Generator().manual_seed(seed)
    caches = [torch.randn((p["n_blocks"], 2, bs, 24), generator=g).to(torch.bfloat16) for _ in range(3)]
    moved = tree_oracle.keep_path([c.float().numpy() for c in caches], p["table"], p["cu"], p["cached"], want[0])
    on_gpu = [c.to(DEV) for c in caches]
    version = on_gpu[0]._version
    attn.keep_path(on_gpu, _ints(p["table"]), arrays[3], arrays[4], kept.path)
    assert on_gpu[0]._version > version
    for c, w in zip(on_gpu, moved):
        assert np.array_equal(c.float().cpu(), w)


class Model:
    """Attention layers with random weights; `step` runs them over whatever tokens are new."""

    def __init__(self, layers=2, hq=4, hkv=2, d=64, vocabulary=11, blocks=256, bs=8):
        g = torch.Generator().manual_seed(0)
        self.hq, self.hkv, self.d, self.bs, width = hq, hkv, d, bs, hq * d
        rand = lambda *s: torch.randn(s, generator=g).to(DEV)
        self.embedding = rand(vocabulary, width)
        self.qkv = [rand(width, (hq + 2 * hkv) * d) / width ** 0.5 for _ in range(layers)]
        self.k, self.v = ([torch.full((blocks, hkv, bs, d), float("nan"), device=DEV) for _ in range(layers)] for _ in range(2))
        self.rotary = attn.rotary_table(512, d)

    def step(self, tokens, slots, positions, attend):
        x = self.embedding[tokens.long()]
        for w, k_cache, v_cache in zip(self.qkv, self.k, self.v):
            q, k, v = (torch.nn.functional.rms_norm(x, x.shape[-1:]) @ w).view(len(x), -1, self.d).split((self.hq, self.hkv, self.hkv), 1)
            q = attn.rope_append(q, k, v, positions, slots, self.rotary, k_cache, v_cache)
            x = x + attend(q, k_cache, v_cache).flatten(1)
        return x @ self.embedding.T


def test_a_server_that_drafts_answers_like_one_that_does_not():
    """Prompts, then steps of drafted trees with blocks that come and go, against one token at a time; fp32, where the two agree on
    the largest logit unless two are within rounding of each other, which is asserted not to happen."""
    torch.manual_seed(1)
    prompts = [[3, 1, 4, 1, 5, 9, 2, 6, 5], [2, 7], [1] * 21]
    batch, want_tokens = len(prompts), 24

    def begin(m):
        free, n_free = _ints(np.random.RandomState(3).permutation(256)), _ints([256])
        table, cached = torch.full((batch, 16), -1, dtype=torch.int32, device=DEV), _ints([0] * batch)
        cu = _ints(np.concatenate([[0], np.cumsum([len(p) for p in prompts])]))
        tokens = _ints(sum(prompts, []))
        s = attn.assign_blocks(m.bs, len(tokens), cu, cached, table, free, n_free)
        logits = m.step(tokens, s.slots, s.positions, lambda q, k, v: attn.attend(q, k, v, s.table, cu, cached))
        last = cu[1:].long() - 1
        return s.table, free, s.counts[:1].clone(), _ints([len(p) for p in prompts]), logits[last]

    # one token at a time
    m = Model()
    table, free, n_free, cached, logits = begin(m)
    chain = [[] for _ in prompts]
    cu = _ints(np.arange(batch + 1))
    for _ in range(want_tokens):
        top = logits.topk(2).values
        assert float((top[:, 0] - top[:, 1]).min()) > 1e-3
        token = logits.argmax(-1).int()
        for c, t in zip(chain, token.tolist()):
            c.append(t)
        s = attn.assign_blocks(m.bs, batch, cu, cached, table, free, n_free)
        logits = m.step(token, s.slots, s.positions, lambda q, k, v: attn.attend(q, k, v, s.table, cu, cached))
        table, n_free, cached = s.table, s.counts[:1].clone(), cached + 1

    # trees: half of the drafted branches go on as the model will, the others by chance
    m = Model()
    table, free, n_free, cached, logits = begin(m)
    rng = random.Random(9)
    said = [[t] for t in logits.argmax(-1).tolist()]
    steps, used = 0, None
    while min(map(len, said)) < want_tokens:
        parents, tokens, cu = [], [], [0]
        for b in range(batch):
            n = rng.choice([1, 4, 11, 19])
            tree = tree_oracle.random_parents(rng, n, 0.7)
            future = chain[b][len(said[b]) - 1:] if len(said[b]) <= want_tokens else []
            line = [said[b][-1]]
            depth = [0]
            for i in range(1, n):
                depth.append(depth[tree[i]] + 1)
                good = depth[i] < len(future) and rng.random() < 0.6
                line.append(future[depth[i]] if good else rng.randrange(11))
            parents += tree
            tokens += line
            cu.append(len(tokens))
        tokens, parents, cu = _ints(tokens), _ints(parents), _ints(cu)
        s = attn.assign_blocks(m.bs, len(tokens), cu, cached, table, free, n_free)
        assert int(s.counts[1]) == 0
        tree = attn.draft_tree(parents, cu, cached, 19)
        logits = m.step(tokens, s.slots, tree.positions,
                        lambda q, k, v: attn.attend_tree(q, k, v, s.table, cu, cached, tree.positions, tree.seen, max_new=19))
        kept = attn.accept_path(tokens, parents, logits.argmax(-1).int(), cu, cached, block_size=m.bs, table=s.table, free_blocks=free, n_free=s.counts[:1])
        attn.keep_path([*m.k, *m.v], s.table, cu, cached, kept.path)
        for b in range(batch):
            path = kept.path[int(cu[b]):int(cu[b]) + int(kept.counts[b])].tolist()
            said[b] += [int(tokens[int(cu[b]) + i]) for i in path[1:]] + [int(kept.next_tokens[b])]
        table, n_free, cached = s.table, kept.n_free, kept.kept_lens
        # blocks in use and free ones are all there are, once each
        held = [int(table[b, e]) for b in range(batch) for e in range(-(-int(cached[b]) // m.bs))]
        assert sorted(held + free[:int(n_free)].tolist()) == list(range(256))
        steps += 1
    for b in range(batch):
        assert said[b][:want_tokens] == chain[b]
    assert steps < want_tokens  # some drafts were kept


def test_a_captured_step_is_replayed():
    """The operators of a step in a graph: lengths, trees and choices change between replays."""
    hq, hkv, d, bs, batch, T = 4, 2, 64, 8, 3, 40
    g = torch.Generator().manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(DEV)
    k, v, q = rand(64, hkv, bs, d), rand(64, hkv, bs, d), rand(T, hq, d)
    cu, cached, parents, tokens, choices = (_ints(np.zeros(n)) for n in (batch + 1, batch, T, T, T))
    table, free, n_free = _ints(np.arange(36).reshape(batch, 12)), _ints(np.arange(64)), _ints([2])

    def step():
        tree = attn.draft_tree(parents, cu, cached, 32)
        out = attn.attend_tree(q, k, v, table, cu, cached, tree.positions, tree.seen, max_new=32)
        kept = attn.accept_path(tokens, parents, choices, cu, cached, block_size=bs, table=table, free_blocks=free, n_free=n_free)
        attn.keep_path([k, v], table, cu, cached, kept.path)
        return tree, out, kept

    def fill(seed):
        rng = random.Random(seed)
        new = [rng.randrange(0, 13) for _ in range(batch)]
        cu.copy_(_ints(np.concatenate([[0], np.cumsum(new)])))
        cached.copy_(_ints([rng.randrange(0, 60) for _ in range(batch)]))
        line = [x for n in new for x in tree_oracle.random_parents(rng, n)]
        parents.copy_(_ints(line + [-1] * (T - len(line))))
        for x in (tokens, choices):
            x.copy_(_ints([rng.randrange(2) for _ in range(T)]))
        return sum(new)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fill(0)
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tree, out, kept = step()
    for seed in range(1, 6):
        n = fill(seed)
        saved = [x.clone() for x in (k, v, free)]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*tree, out[:n], *kept, k, v, free)]
        for x, s in zip((k, v, free), saved):
            x.copy_(s)
        tree_e, out_e, kept_e = step()
        for a, b in zip(got, (*tree_e, out_e[:n], *kept_e, k, v, free)):
            assert torch.equal(a, b)


def test_on_another_stream():
    p = th.make(2, *th.CASES["chunk_group"])
    want = _attend(p)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _attend(p)
    assert np.array_equal(want[0], got[0]) and np.array_equal(want[1], got[1])


def test_rows_of_no_sequence_stay_as_they_are():
    p = th.make(6, *th.CASES["chunk"])
    out = torch.full((p.T + 5, p.hq, p.d), 7.0, dtype=torch.bfloat16, device=DEV)
    pad = lambda x: torch.cat([x, x[:5]])
    got = attn.attend_tree(pad(p.q.to(DEV)), p.k_cache.to(DEV), p.v_cache.to(DEV), _ints(p.table), _ints(p.cu), _ints(p.cached), pad(_ints(p.positions)),
                           pad(_ints(p.bits)), out=out)
    assert got.data_ptr() == out.data_ptr() and bool((out[p.T:] == 7.0).all())
    assert np.array_equal(out[:p.T].cpu().double().numpy(), _attend(p)[0])


@pytest.mark.parametrize("new", [[3, 2], [17, 40], [300]])
def test_caches_beyond_32_bits(new):
    """Blocks whose elements lie behind 2^32: the same results, bit for bit, as in a small cache."""
    p = th.make(31, 8, 2, 128, 16, "bf16", new, [100 + 7 * b for b in range(len(new))], max_new=max(new))
    small = [p.k_cache.to(DEV), p.v_cache.to(DEV)]
    n, blocks = small[0].shape[0], (1 << 32) // (2 * 16 * 128) + 50
    caches = [torch.empty(blocks, 2, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in small]
    for c, s in zip(caches, small):
        c[blocks - n:] = s
    table = np.asarray(p.table)
    args = (_ints(p.cu), _ints(p.cached), _ints(p.positions), _ints(p.bits))
    far = _ints(np.where(table >= 0, table + blocks - n, table))
    a, b = (attn.attend_tree(p.q.to(DEV), *c, t, *args, scale=p.scale, max_new=p.max_new) for c, t in ((small, _ints(table)), (caches, far)))
    assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    path = _ints(np.concatenate([np.minimum(2 * np.arange(m), m - 1) if m < 3 else np.concatenate([np.arange(0, m, 2), np.full(m // 2, -1)]) for m in new]))
    for c, t in ((small, _ints(table)), (caches, far)):
        attn.keep_path(c, t, args[0], args[1], path)
    bits = lambda t: t.view(torch.int16)  # (rows that hold no key are NaN)
    assert all(torch.equal(bits(c[blocks - n:]), bits(s)) for c, s in zip(caches, small))


def test_no_tokens():
    none, cu, one = _ints([]), _ints([0, 0]), _ints([3])
    tree = attn.draft_tree(none, cu, one, 5)
    assert tree.positions.shape == (0,) and tree.seen.shape == (0, 1)
    cache = torch.zeros(2, 2, 16, 64, device=DEV)
    out = attn.attend_tree(torch.zeros(0, 2, 64, device=DEV), cache, cache, _ints([[0]]), cu, one, *tree)
    assert out.shape == (0, 2, 64)
    kept = attn.accept_path(none, none, none, cu, one)
    assert [x.tolist() for x in kept[:4]] == [[], [0], [-1], [3]]
    attn.keep_path([cache, cache.clone()], _ints([[0]]), cu, one, kept.path)
    attn.keep_path([], _ints([[0]]), cu, one, kept.path)


def test_no_sequences():
    """The free list stays as long as it is."""
    none, cu = _ints([]), _ints([0])
    free = _ints([5, 6, 7, -1])
    kept = attn.accept_path(none, none, none, cu, none, block_size=16, table=torch.zeros(0, 4, dtype=torch.int32, device=DEV), free_blocks=free, n_free=_ints([3]))
    assert [x.tolist() for x in kept] == [[], [], [], [], [3]] and free.tolist() == [5, 6, 7, -1]
    assert attn.accept_path(none, none, none, cu, none).n_free is None
    tree = attn.draft_tree(none, cu, none, 3)
    assert tree.positions.shape == (0,) and tree.seen.shape == (0, 1)
    attn.keep_path([torch.zeros(2, 2, 16, 64, device=DEV)], torch.zeros(0, 4, dtype=torch.int32, device=DEV), cu, none, none)


def test_refusals():
    ints, cu, one = _ints([-1, 0]), _ints([0, 2]), _ints([3])
    q, cache = torch.zeros(2, 2, 64, device=DEV), torch.zeros(2, 2, 16, 64, device=DEV)
    table, seen = _ints([[0, 1]]), _ints([[1], [3]])
    good = (q, cache, cache.clone(), table, cu, one, ints, seen)
    attn.attend_tree(*good)
    for at, bad in ((6, ints[:1]), (6, ints.long()), (7, seen[:1]), (7, seen.t()), (7, _ints(np.zeros((2, 0)))), (7, _ints(np.zeros((2, 33)))), (0, q.half())):
        with pytest.raises((ValueError, attn.AttnError)):
            attn.attend_tree(*good[:at], bad, *good[at + 1:])
    for most in (0, 1025, -3):
        with pytest.raises(ValueError, match="max_new"):
            attn.draft_tree(ints, cu, one, most)
    with pytest.raises(attn.AttnError, match="window"):
        attn.draft_tree(ints, cu, one, 2, window=-1)
    with pytest.raises(ValueError, match="together"):
        attn.accept_path(ints, ints, ints, cu, one, table=table, block_size=16)
    with pytest.raises(attn.AttnError, match="power of two"):
        attn.accept_path(ints, ints, ints, cu, one, table=table, block_size=12, free_blocks=ints, n_free=one)
    path = _ints([0, -1])
    for bad in ([cache, cache], [cache, cache.view(-1)[:2048].view(1, 2, 16, 64)], [cache, cache.half()], [cache.transpose(1, 2)], [cache.cpu()]):
        with pytest.raises((ValueError, attn.AttnError)):
            attn.keep_path(bad, table, cu, one, path)
    with pytest.raises(TypeError):
        attn.keep_path(cache, table, cu, one, path)
    with pytest.raises(ValueError, match="requires grad"):
        attn.keep_path([cache.clone().requires_grad_()], table, cu, one, path)
    with pytest.raises(ValueError, match="q requires grad"):
        attn.attend_tree(q.clone().requires_grad_(), *good[1:])
