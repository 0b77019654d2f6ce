"""The gated recurrence on the GPU: against its definition in 64 bits, its gradients against the chain rule and against differences,
captured into graphs, on another stream, two calls at once, and with the attention layers' operators in a step of drafted trees."""
from __future__ import annotations

import random

import numpy as np
import pytest
import torch

import rec_helpers as rh
import rec_oracle
import tree_oracle
from paper_2411_19379_amd import attention as attn
from paper_2411_19379_amd import recurrence as rec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _on_gpu(p, gates_apart=True):
    """x, r, i, decay, bounds and initial states; r and i as parts of one projection's rows."""
    x, decay = p.x.to(DEV), p.decay.to(DEV)
    if gates_apart:
        r, i = p.r.to(DEV), p.i.to(DEV)
    else:
        both = torch.cat([p.r, p.i], 1).to(DEV)
        r, i = both[:, :p.C], both[:, p.C:]
    return x, r, i, decay, _ints(p.cu), None if p.init is None else p.init.to(DEV)


def _numpy(*all_):
    return [None if t is None else t.detach().double().cpu().numpy() for t in all_]


SIZES = dict(rh.CASES)
SIZES.update(long=(192, "bf16", [5000, 1], {}), wide=(2560, "bf16", [300, 129, 0, 64], {}), wide_odd=(1001, "f16", [500, 70], {}),
             many=(128, "f32", [37] * 60 + [0] * 5, dict(init=False)), two=(2560, "bf16", [900, 300, 0, 64], {}), two_f32=(2048, "f32", [1300], {}),
             two_f16=(1000, "f16", [2500, 3], dict(init=False)))


@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("name", sorted(SIZES))
def test_scan(name, apart):
    C, dtype, lens, more = SIZES[name]
    p = rh.make(15, C, dtype, lens, **more)
    x, r, i, decay, cu, init = _on_gpu(p, apart)
    ckpt = [0, p.T - 1, p.T // 2, p.T // 3, p.T // 2, -1, p.T + 5, 2 ** 31 - 1]
    out = rec.gated_scan(x, r, i, decay, cu, init_states=init, ckpt=_ints(ckpt))
    rh.check_scan(p, *_numpy(out.y, out.final), ckpt, *_numpy(out.ckpt_states))
    again = rec.gated_scan(x, r, i, decay, cu, init_states=init)
    inside = slice(int(p.cu[0]), int(p.cu[-1]))
    assert again.ckpt_states is None and torch.equal(out.y[inside], again.y[inside]) and torch.equal(out.final, again.final)


@pytest.mark.parametrize("name", sorted(SIZES))
def test_grads(name):
    C, dtype, lens, more = SIZES[name]
    p = rh.make(16, C, dtype, lens, **more)
    x, r, i, decay, cu, init = _on_gpu(p, False)
    dy, d_final = p.dy.to(DEV), p.d_final.to(DEV)
    got = rec.gated_scan_grads(dy, d_final, x, r, i, decay, cu, init_states=init)
    rh.check_grads(p, _numpy(*got))
    leaves = [t.clone().requires_grad_() for t in (x, r.contiguous(), i.contiguous(), decay) + (() if init is None else (init,))]
    out = rec.gated_scan(*leaves[:4], cu, init_states=leaves[4] if init is not None else None)
    for a, b in zip(torch.autograd.grad((out.y, out.final), leaves, (dy, d_final)), got):
        assert torch.equal(a, b)


def test_resumed_pieces_are_the_whole():
    """A prompt in three calls that resume from the state behind the one in front: bit for bit where the pieces are whole chunks
    of a group, within the bounds elsewhere."""
    p = rh.make(3, 256, "bf16", [1500])
    x, r, i, decay, cu, init = _on_gpu(p)
    for cuts in ([0, 512, 1024, 1500], [0, 1, 700, 1500]):
        states, parts = init, []
        for a, b in zip(cuts, cuts[1:]):
            out = rec.gated_scan(x[a:b], r[a:b], i[a:b], decay, _ints([0, b - a]), init_states=states)
            parts.append(out.y)
            states = out.final
        rh.check_scan(p, *_numpy(torch.cat(parts), states))


def test_gradients_against_differences():
    p = rh.make(1, 3, "f32", [9, 4], keep=(0.6, 0.9))
    values = [v.double().numpy() for v in (p.x, p.r, p.i, p.decay, p.init)]

    def loss(x, r, i, decay, init):
        h, final = rec_oracle.scan(x, r, i, decay, p.cu, p.sharpness, init)
        return float((h * p.dy.double().numpy()).sum() + (final * p.d_final.double().numpy()).sum())

    x, r, i, decay, cu, init = _on_gpu(p)
    got = _numpy(*rec.gated_scan_grads(p.dy.to(DEV), p.d_final.to(DEV), x, r, i, decay, cu, init_states=init))
    step = 1e-5
    for k, g in enumerate(got):
        for at in np.ndindex(*values[k].shape):
            up, down = ([v.copy() for v in values] for _ in range(2))
            up[k][at] += step
            down[k][at] -= step
            # central differences: an error of step^2 times a third derivative of at most some hundreds
            assert abs((loss(*up) - loss(*down)) / (2 * step) - g[at]) < 1e-4 * (1 + abs(g[at]))


def test_graph_of_gradients():
    p = rh.make(5, 64, "bf16", [70, 20])
    x, r, i, decay, cu, init = _on_gpu(p)
    decay.requires_grad_()
    out = rec.gated_scan(x, r, i, decay, cu, init_states=init)
    out.y.sum().backward()  # a gradient that is expanded from one value
    want = rec.gated_scan_grads(torch.ones_like(x), None, x, r, i, decay, cu, init_states=init)
    assert torch.equal(decay.grad, want.decay) and x.grad is None
    decay.grad = None
    out = rec.gated_scan(x, r, i, decay, cu, init_states=init)
    out.final.square().sum().backward()
    want = rec.gated_scan_grads(None, 2 * out.final.detach(), x, r, i, decay, cu, init_states=init)
    assert torch.equal(decay.grad, want.decay)
    # gradients that have strides of their own
    out = rec.gated_scan(x, r, i, decay, cu)
    dy = torch.randn(64, 90, device=DEV).bfloat16().t()
    a, = torch.autograd.grad(out.y, decay, dy)
    assert torch.equal(a, rec.gated_scan_grads(dy.contiguous(), None, x, r, i, decay, cu).decay)
    # an input that has changed since, and gradients of gradients
    out = rec.gated_scan(x, r, i, decay, cu)
    x.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        out.y.sum().backward()
    out = rec.gated_scan(x, r, i, decay, cu)
    g, = torch.autograd.grad(out.y.float().square().sum(), decay, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_step_and_tree():
    for C, dtype, batch in ((4096, "bf16", 5), (65, "f32", 3), (7, "f16", 1)):
        p = rh.make(4, C, dtype, [1] * batch)
        x, r, i, decay, _, states = _on_gpu(p, False)
        version = states._version
        y = rec.gated_step(x, r, i, decay, states)
        assert states._version > version
        rh.check_scan(p, *_numpy(y, states))
    for C, dtype, lens in ((2560, "bf16", [17, 0, 64, 3]), (33, "f16", [200, 1]), (128, "f32", [70])):
        p = rh.make(4, C, dtype, lens)
        rng = random.Random(C)
        parents = np.array([q for n in lens for q in tree_oracle.random_parents(rng, n, 0.6, 0.1)], np.int32)
        x, r, i, decay, cu, states = _on_gpu(p, False)
        y, nodes = rec.gated_step_tree(x, r, i, decay, states, cu, _ints(parents))
        assert torch.equal(y, nodes.to(y.dtype)) and torch.equal(states.cpu(), p.init)
        # every branch is a sequence of its own
        for b, n in enumerate(lens):
            for k in {0, n // 2, n - 1} if n else ():
                line = [int(p.cu[b]) + a for a in tree_oracle.branch(parents[p.cu[b]:p.cu[b + 1]].tolist(), k)[::-1]]
                q = rh.make(0, C, dtype, [len(line)])
                q.x, q.r, q.i, q.decay, q.init = p.x[line], p.r[line], p.i[line], p.decay, p.init[b:b + 1]
                rh.check_scan(q, *_numpy(y[line], nodes[line[-1:]]))
        path, counts = torch.full((p.T,), -1, dtype=torch.int32, device=DEV), _ints([min(n, 2) for n in lens])
        for b, n in enumerate(lens):
            path[int(p.cu[b]):int(p.cu[b]) + min(n, 2)] = _ints([0, n - 1][:n])
        rec.keep_states(states, nodes, cu, path, counts)
        for b, n in enumerate(lens):
            assert torch.equal(states[b], nodes[int(p.cu[b]) + (n - 1 if n > 1 else 0)] if n else p.init[b].to(DEV))


def test_a_step_of_trees_keeps_what_a_chain_would_have():
    """Drafted trees through the recurrence and the choice of a branch, step after step, against the chain of the kept tokens."""
    C, batch, vocabulary = 128, 3, 5
    g = torch.Generator().manual_seed(2)
    embedding = torch.randn(vocabulary, 3 * C, generator=g).to(DEV)
    decay = torch.full((C,), -5.0, device=DEV)
    rng = random.Random(4)
    states, chain = torch.zeros(batch, C, device=DEV), [[] for _ in range(batch)]
    cached = _ints([0] * batch)
    for _ in range(6):
        lens = [rng.choice([1, 7, 30]) for _ in range(batch)]
        cu = _ints(np.concatenate([[0], np.cumsum(lens)]))
        parents = _ints([q for n in lens for q in tree_oracle.random_parents(rng, n, 0.7)])
        tokens, choices = (torch.randint(vocabulary, (sum(lens),), generator=g).int().to(DEV) for _ in range(2))
        x, r, i = embedding[tokens.long()].split(C, 1)
        y, nodes = rec.gated_step_tree(x, r, i, decay, states, cu, parents)
        kept = attn.accept_path(tokens, parents, choices, cu, cached)
        rec.keep_states(states, nodes, cu, kept.path, kept.counts)
        cached = kept.kept_lens
        for b in range(batch):
            at = int(cu[b])
            chain[b] += [int(tokens[at + k]) for k in kept.path[at:at + int(kept.counts[b])].tolist()]
    assert max(map(len, chain)) > 6
    for b in range(batch):
        rows = embedding[torch.tensor(chain[b], device=DEV)]
        x, r, i = rows.split(C, 1)
        q = rh.make(0, C, "f32", [len(chain[b])], init=False)
        q.x, q.r, q.i, q.decay = x.cpu(), r.cpu(), i.cpu(), decay.cpu()
        rh.check_scan(q, rec.gated_scan(x, r, i, decay, _ints([0, len(chain[b])])).y.double().cpu().numpy(), _numpy(states[b:b + 1])[0])


def test_captured_and_replayed():
    """Scan, gradients and steps in a graph: bounds, inputs and states change between replays."""
    C, T, batch = 192, 1300, 4
    g = torch.Generator().manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=g).to(DEV)
    x, r, i, dy = (rand(T, C).bfloat16() for _ in range(4))
    decay, init, d_final, states = rand(C) - 5, rand(batch, C), rand(batch, C), rand(batch, C)
    cu, ckpt, parents = _ints([0] * (batch + 1)), _ints([0, 0, 0]), _ints([-1] * T)

    def step():
        out = rec.gated_scan(x, r, i, decay, cu, init_states=init, ckpt=ckpt)
        grads = rec.gated_scan_grads(dy, d_final, x, r, i, decay, cu, init_states=init)
        y, nodes = rec.gated_step_tree(x, r, i, decay, states, cu, parents)
        y1 = rec.gated_step(x[:batch], r[:batch], i[:batch], decay, states)
        return [*out, *grads, y1], [y, nodes]

    def fill(seed):
        rng = random.Random(seed)
        cuts = sorted(rng.randrange(T + 1) for _ in range(batch))
        cu.copy_(_ints([0] + cuts))
        ckpt.copy_(_ints([rng.randrange(T) for _ in range(3)]))
        parents.copy_(_ints([rng.randrange(-1, 40) for _ in range(T)]))
        x.normal_()
        return cuts[-1]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fill(0)
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in range(1, 6):
        n = fill(seed)
        before = states.clone()
        graph.replay()
        torch.cuda.synchronize()
        first, rows = [t.clone() for t in captured[0]], [t[:n].clone() for t in captured[1]]
        after = states.clone()
        states.copy_(before)
        eager = step()
        first[0], eager[0][0] = first[0][:n], eager[0][0][:n]  # (y: rows of no sequence are not written)
        for a, b in zip((*first, *rows, after), (*eager[0], *(t[:n] for t in eager[1]), states)):
            assert torch.equal(a, b)


def test_a_graph_of_gradients_is_not_captured():
    p = rh.make(5, 64, "bf16", [70])
    x, r, i, decay, cu, _ = _on_gpu(p)
    decay.requires_grad_()
    graph = torch.cuda.CUDAGraph()
    y = torch.zeros(1, device=DEV)
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="not captured"):
            rec.gated_scan(x, r, i, decay, cu)
        y += 1
    graph.replay()
    assert float(y) == 1.0


def test_two_calls_at_once():
    """Calls on two streams have workspaces of their own."""
    p = rh.make(7, 512, "bf16", [3000, 40])
    args = _on_gpu(p)
    want = rec.gated_scan(*args[:5], init_states=args[5])
    grads = rec.gated_scan_grads(p.dy.to(DEV), None, *args[:5], init_states=args[5])
    dy = p.dy.to(DEV)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append((rec.gated_scan(*args[:5], init_states=args[5]), rec.gated_scan_grads(dy, None, *args[:5], init_states=args[5])))
    torch.cuda.synchronize()
    for a, b in outs:
        assert torch.equal(a.y, want.y) and torch.equal(a.final, want.final)
        assert all(torch.equal(u, v) for u, v in zip(b, grads))


@pytest.mark.parametrize("name", ["two", "two_f32", "two_f16", "long"])
def test_unaligned_rows_have_the_same_results(name):
    C, dtype, lens, more = SIZES[name]
    p = rh.make(12, C, dtype, lens, **more)
    x, r, i, decay, cu, init = _on_gpu(p)
    inside = slice(int(p.cu[0]), int(p.cu[-1]))
    moved = torch.empty(p.T * C + 1, dtype=x.dtype, device=DEV)[1:].view(p.T, C).copy_(x)
    a, b = (rec.gated_scan(t, r, i, decay, cu, init_states=init) for t in (x, moved))
    assert torch.equal(a.y[inside], b.y[inside]) and torch.equal(a.final, b.final)
    dy = p.dy.to(DEV)
    for a, b in zip(*(rec.gated_scan_grads(dy, None, t, r, i, decay, cu, init_states=init) for t in (x, moved))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("C,dtype", [(70, "bf16"), (128, "f32"), (33, "f16")])
def test_in_place(C, dtype):
    """y in the place of an input, and the final states in that of the initial ones."""
    p = rh.make(9, C, dtype, [400, 0, 3, 130])
    x, r, i, decay, cu, init = _on_gpu(p)
    inside = slice(int(p.cu[0]), int(p.cu[-1]))
    states = torch.randn(p.T, C, device=DEV)
    parents = _ints(np.concatenate([np.full(int(p.cu[0]), -1)] + [np.arange(n) // 2 - 1 for n in p.lens] + [np.full(p.T - int(p.cu[-1]), -1)]))
    for at in range(3):
        def arguments():
            args = [t.clone() for t in (x, r, i)]
            return args, args[at]
        args, out = arguments()
        want = rec.gated_scan(*args, decay, cu, init_states=init)
        got = rec.gated_scan(*args, decay, cu, init_states=init, out=out)
        assert got.y is out and torch.equal(out[inside], want.y[inside]) and torch.equal(got.final, want.final)
        args, out = arguments()
        y, nodes = rec.gated_step_tree(*args, decay, init, cu, parents)
        again, same = rec.gated_step_tree(*args, decay, init, cu, parents, out=out)
        assert torch.equal(again[inside], y[inside]) and torch.equal(same[inside], nodes[inside])
        args, out = arguments()
        one, two = states.clone(), states.clone()
        y = rec.gated_step(*args, decay, one)
        assert torch.equal(rec.gated_step(*args, decay, two, out=out), y) and torch.equal(one, two)
    both, y, shape = init.clone(), torch.empty_like(x), rec.RecShape(C, rh.CODE[dtype], 8.0)
    ws = torch.empty(rec.rec_workspace_bytes(shape, len(p.lens), p.T), dtype=torch.uint8, device=DEV)
    want = rec.gated_scan(x, r, i, decay, cu, init_states=init)
    rows = [v for t in (x, r, i) for v in (t.data_ptr(), C)]
    rc = rec.load_library().rec_scan(shape, len(p.lens), p.T, *rows, decay.data_ptr(), cu.data_ptr(), both.data_ptr(), None, 0, y.data_ptr(), C,
                                     both.data_ptr(), None, None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(both, want.final) and torch.equal(y[inside], want.y[inside])


def test_gradients_that_are_far_apart_or_expanded():
    p = rh.make(6, 40, "bf16", [3])
    x, r, i, decay, cu, _ = _on_gpu(p)
    want = rec.gated_scan_grads(torch.ones_like(x), None, x, r, i, decay, cu)
    wide = torch.ones(p.T, rec.REC_MOST_STRIDE + 8, device=DEV, dtype=x.dtype)[:, :p.C]
    for dy in (wide, torch.ones(1, 1, device=DEV, dtype=x.dtype).expand(p.T, p.C)):
        leaf = x.clone().requires_grad_()
        rec.gated_scan(leaf, r, i, decay, cu).y.backward(dy)
        assert torch.equal(leaf.grad, want.x)


def test_tensors_beyond_32_bits():
    """2^31 elements and some rows: the last sequences as in a batch of their own."""
    C, n = 4096, 300
    T = (1 << 31) // C + 200
    g = torch.Generator(DEV).manual_seed(4)
    tail = [torch.randn(n, C, device=DEV, generator=g).bfloat16() for _ in range(3)]
    x = torch.zeros(T, C, dtype=torch.bfloat16, device=DEV)
    r, i = torch.zeros_like(x), torch.zeros_like(x)
    for whole, part in zip((x, r, i), tail):
        whole[T - n:] = part
    decay, init = torch.randn(C, device=DEV, generator=g), torch.randn(3, C, device=DEV, generator=g)
    cu, own = _ints([0, T - n, T - 100, T]), _ints([0, n - 100, n])
    want, got = rec.gated_scan(*tail, decay, own, init_states=init[1:], ckpt=_ints([n - 2])), rec.gated_scan(x, r, i, decay, cu, init_states=init, ckpt=_ints([T - 2]))
    # Chunks fall elsewhere, so maps are composed in another order.  A token's step costs a state at most 32 half-steps of 2^-24 of the
    # largest one: the sum's 1, those of a (exponent, its argument's relative to |log a| a <= 1/e, the composed product) 11, and 10 of
    # the added term, which is at most twice the largest state.  Both sides are that far off after at most n tokens.
    apart = 2 * n * 32 * 2.0 ** -24
    assert float((got.ckpt_states - want.ckpt_states).abs().max()) <= apart * float(want.y.float().abs().max())
    assert float((got.final[1:] - want.final).abs().max()) <= apart * float(want.y.float().abs().max())
    # a step of bf16 where that decides a rounding
    assert float((got.y[T - n:].float() - want.y.float()).abs().max()) <= 2.0 ** -7 * float(want.y.float().abs().max())
    parents = _ints(np.concatenate([np.full(T - n, -1), np.arange(n - 100) - 1, np.arange(100) // 2 - 1]))
    y, nodes = rec.gated_step_tree(x, r, i, decay, init, cu, parents)
    want_y, want_nodes = rec.gated_step_tree(*tail, decay, init[1:], own, parents[T - n:].contiguous())
    assert torch.equal(y[T - n:], want_y) and torch.equal(nodes[T - n:], want_nodes)
    del y, nodes
    dy = torch.zeros_like(x)
    dy[T - n:] = tail[1]
    a, b = rec.gated_scan_grads(dy, None, x, r, i, decay, cu, init_states=init), rec.gated_scan_grads(tail[1], None, *tail, decay, own, init_states=init[1:])
    for u, v in zip(a[:3], b[:3]):
        assert float((u[T - n:].float() - v.float()).abs().max()) <= 2.0 ** -7 * float(v.float().abs().max()) and float(u[:T - n].abs().max()) == 0.0


def test_no_tokens():
    x, decay, states = torch.zeros(0, 6, device=DEV), torch.zeros(6, device=DEV), torch.randn(2, 6, device=DEV)
    cu = _ints([0, 0, 0])
    out = rec.gated_scan(x, x, x, decay, cu, init_states=states, ckpt=_ints([0]))
    assert out.y.shape == (0, 6) and torch.equal(out.final, states) and torch.equal(out.ckpt_states, torch.zeros(1, 6, device=DEV))
    assert torch.equal(rec.gated_scan(x, x, x, decay, cu).final, torch.zeros(2, 6, device=DEV))
    got = rec.gated_scan_grads(x, states, x, x, x, decay, cu)
    assert got.x.shape == (0, 6) and torch.equal(got.decay, torch.zeros(6, device=DEV)) and torch.equal(got.init_states, states)
    y, nodes = rec.gated_step_tree(x, x, x, decay, states, cu, _ints([]))
    assert y.shape == nodes.shape == (0, 6)
    rec.keep_states(states, nodes, cu, _ints([]), _ints([0, 0]))
    assert rec.gated_step(x, x, x, decay, states[:0]).shape == (0, 6)


def test_refusals():
    x, decay, states, cu = torch.zeros(4, 6, device=DEV), torch.zeros(6, device=DEV), torch.zeros(2, 6, device=DEV), _ints([0, 1, 4])
    rec.gated_scan(x, x, x, decay, cu, init_states=states)
    for bad in (x.double(), x[:, :5], x[:3], x.t().contiguous().t(), x.cpu(), x[None], x[:1].expand(4, 6)):
        for at in range(3):
            with pytest.raises((ValueError, rec.RecError)):
                rec.gated_scan(*[bad if k == at else x for k in range(3)], decay, cu)
    for kw in (dict(init_states=states[:1]), dict(init_states=states.half()), dict(sharpness=0.0), dict(sharpness=float("inf")), dict(sharpness=float("nan")),
               dict(ckpt=cu.long()), dict(out=x.half()), dict(out=x[:3])):
        with pytest.raises((ValueError, rec.RecError)):
            rec.gated_scan(x, x, x, decay, cu, **kw)
    for bad in (decay.half(), decay[:5], decay.cpu()):
        with pytest.raises(ValueError):
            rec.gated_scan(x, x, x, bad, cu)
    for bad in (cu.long(), cu[:0], cu.cpu()):
        with pytest.raises(ValueError):
            rec.gated_scan(x, x, x, decay, bad)
    leaf = x.clone().requires_grad_()
    for kw in (dict(ckpt=_ints([0])), dict(out=x.clone())):
        with pytest.raises(ValueError, match="not differentiable"):
            rec.gated_scan(leaf, x, x, decay, cu, **kw)
    with pytest.raises(ValueError, match="out requires grad"):
        rec.gated_scan(x, x, x, decay, cu, out=x.clone().requires_grad_())
    with pytest.raises(ValueError, match="x requires grad"):
        rec.gated_step(leaf[:2], x[:2], x[:2], decay, states)
    with pytest.raises(ValueError, match="states requires grad"):
        rec.gated_step_tree(x, x, x, decay, states.clone().requires_grad_(), cu, _ints([-1] * 4))
    with pytest.raises(ValueError):
        rec.gated_step(x, x, x, decay, states)
    with pytest.raises(ValueError):
        rec.gated_step_tree(x, x, x, decay, states, cu, _ints([-1] * 3))
    with pytest.raises(ValueError):
        rec.keep_states(states, x, cu, _ints([0] * 3), _ints([1, 1]))
