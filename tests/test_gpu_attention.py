"""The attention operators on the GPU, through the Python entry points, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import attn_helpers as ah
import attn_oracle
from test_attention_emulation import ASSIGN, CASES, MANY, NOT_FINITE, PADDED, ROPE, check_padded, many, padded, rope_check, rope_problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _attend(p, **kw):
    from paper_2411_19379_amd import attention as attn
    out, lse = attn.attend(p.q.to(DEV), p.k_cache.to(DEV), p.v_cache.to(DEV), _dev(p.table), _dev(p.cu), _dev(np.array(p.cached, np.int32)),
                           scale=p.scale, window=p.window, sinks=p.sinks, max_new=p.max_new, return_lse=True, **kw)
    return out.double().cpu().numpy(), lse.cpu().numpy()


@pytest.mark.parametrize("name", sorted(CASES))
def test_attend_small(name):
    print(f"attend {name}", flush=True)
    p = ah.make(11, *CASES[name])
    ah.check(p, *_attend(p), name)


@pytest.mark.parametrize("name", ["decode", "few_window", "chunk", "chunk_window", "f32_wide_window"])
def test_attend_with_blocks_missing(name):
    print(f"attend holes {name}", flush=True)
    p = ah.make(5, *CASES[name], holes=0.5)
    ah.check(p, *_attend(p), name)


@pytest.mark.parametrize("name", ["decode", "few_window", "chunk", "f32"])
def test_attend_with_a_table_that_is_too_narrow(name):
    print(f"attend narrow table {name}", flush=True)
    p = ah.make(13, *CASES[name])
    for width in (1, 3):
        p.table = np.ascontiguousarray(ah.make(13, *CASES[name]).table[:, :width])
        ah.check(p, *_attend(p), f"{name} {width}")


@pytest.mark.parametrize("where", ["v", "k"])
@pytest.mark.parametrize("name", NOT_FINITE)
def test_attend_not_finite(name, where):
    print(f"attend not finite {name} {where}", flush=True)
    p = ah.make(7, *CASES[name])
    cache = p.v_cache if where == "v" else p.k_cache
    for i, bad in enumerate([float("inf"), float("nan"), -float("inf")]):
        seq = max(range(len(p.new)), key=lambda b: p.new[b])
        total = p.new[seq] + p.cached[seq]
        for j in {total - 1 - 2 * i, total // 2 + i, total * 3 // 4 - i}:
            if 0 <= j < total:
                block, row = p.block_row(seq, j)
                cache[block, i % p.hkv, row, (5 * i + j) % p.d] = bad
    ah.check(p, *_attend(p), name)


def _reference64(p):
    """The definition with torch in 64 bits on the GPU, for lengths the plain oracle takes too long for."""
    T, hq, d, g = p.T, p.hq, p.d, p.hq // p.hkv
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(out)
    lse = torch.full((T, hq), -float("inf"), dtype=torch.float64, device=DEV)
    for b in range(len(p.new)):
        n, c = p.new[b], p.cached[b]
        if n == 0:
            continue
        j = torch.arange(n + c, device=DEV)
        blocks = _dev(p.table[b]).long()[j // p.bs]
        there = (blocks >= 0) & (blocks < p.k_cache.shape[0])
        blocks = blocks.clamp(0, p.k_cache.shape[0] - 1)
        k = p.k_cache.to(DEV)[blocks, :, j % p.bs].double()
        v = p.v_cache.to(DEV)[blocks, :, j % p.bs].double()
        k[~there] = 0
        v[~there] = 0
        pos = torch.arange(c, c + n, device=DEV)[:, None]
        seen = (j <= pos) & there
        if p.window:
            seen &= (j > pos - p.window) | (j < p.sinks)
        for h in range(hq):
            s = p.q[p.cu[b]:p.cu[b + 1], h].to(DEV).double() @ k[:, h // g].T * p.scale
            s[~seen] = -float("inf")
            some = seen.any(1)
            w = torch.softmax(s, 1)
            w[~some] = 0
            rows = slice(int(p.cu[b]), int(p.cu[b + 1]))
            out[rows, h] = w @ v[:, h // g]
            size[rows, h] = w @ v[:, h // g].abs()
            lse[rows, h] = torch.logsumexp(s, 1)
    return out.cpu().numpy(), lse.cpu().numpy(), size.cpu().numpy()


# heads, key heads, head_dim, block size, type, new tokens, cached tokens, window, sinks, max_new
LONG = {
    "decode_long": (8, 2, 128, 16, "bf16", [1] * 5, [9000, 1, 4096, 333, 20000], 0, 0, 1),
    "decode_long_f16_window": (8, 8, 64, 32, "f16", [1] * 4, [9000, 1, 4097, 333], 1000, 4, 1),
    "speculative": (8, 2, 128, 64, "bf16", [5, 3, 1, 8], [5000, 17, 4096, 333], 0, 0, 8),
    "speculative_wide": (32, 2, 64, 16, "f16", [4, 2], [3000, 170], 0, 0, 4),
    "chunk_over_long": (4, 1, 128, 16, "bf16", [137], [6000], 0, 0, 137),
    "mixed": (8, 2, 128, 16, "f16", [1, 300, 1, 0, 77, 2], [2000, 100, 1, 5, 1500, 64], 0, 0, 0),
    "mixed_window": (6, 2, 64, 8, "bf16", [1, 300, 1, 0, 777, 2], [2000, 100, 1, 5, 1500, 64], 200, 70, 0),
    "prompt": (4, 2, 128, 32, "bf16", [2100], [0], 0, 0, 0),
    "prompt_f16_small_heads": (6, 3, 64, 16, "f16", [1500, 900], [64, 63], 0, 0, 0),
    "f32_long": (4, 2, 128, 16, "f32", [1, 200], [5000, 700], 0, 0, 0),
}


@pytest.mark.parametrize("name", sorted(LONG))
def test_attend_long(name):
    print(f"attend {name}", flush=True)
    p = ah.make(21, *LONG[name])
    ah.check(p, *_attend(p), name, ref=_reference64(p))


# One long sequence among many short ones: a tile for every workgroup, and some of them cut into many pieces all the same.
SKEWED = {
    "chunks": (8, 8, 64, 16, "bf16", [200] * 40 + [100] + [30] * 5, [7] * 20 + [0] * 20 + [20000] + [64] * 5, 0, 0, 0),
    "chunks_hint": (8, 8, 128, 32, "f16", [20] * 64 + [17], [100] * 64 + [20000], 0, 0, 20),
    "tokens": (4, 4, 128, 16, "bf16", [1] * 300, [10 + i % 50 for i in range(299)] + [40000], 0, 0, 1),
    "tokens_window": (4, 4, 64, 16, "f16", [1] * 300, [10 + i % 50 for i in range(299)] + [40000], 3000, 5, 1),
    "f32": (8, 8, 64, 16, "f32", [60] * 130 + [3], [7] * 130 + [9000], 0, 0, 0),
}


@pytest.mark.parametrize("name", sorted(SKEWED))
def test_attend_one_long_sequence_among_many(name):
    print(f"attend skewed {name}", flush=True)
    p = ah.make(23, *SKEWED[name])
    ah.check(p, *_attend(p), name, ref=_reference64(p))


def _random(seed):
    rs = np.random.RandomState(seed)
    hkv, group = int(rs.choice([1, 2, 3, 8])), int(rs.choice([1, 2, 3, 4, 7, 16, 33]))
    batch, longest = int(rs.choice([1, 2, 5, 17, 70])), int(rs.choice([1, 1, 4, 40, 400]))
    new = [int(rs.randint(0, longest + 1)) for _ in range(batch)]
    new[int(rs.randint(batch))] = longest
    cached = [int(rs.choice([0, 1, 15, 16, 63, 64, 65, int(rs.randint(0, 900)), int(rs.randint(0, 4000))])) for _ in range(batch)]
    window = int(rs.choice([0, 0, 1, 31, 200, 1000]))
    return (group * hkv, hkv, int(rs.choice([64, 128])), int(rs.choice([1, 2, 4, 8, 16, 32, 64, 256])), str(rs.choice(["f32", "bf16", "f16"])), new, cached,
            window, int(rs.choice([0, 1, 5, 40])) if window else 0, int(rs.choice([0, longest])))


@pytest.mark.parametrize("seed", range(40))
def test_attend_random(seed):
    """Heads, lengths, blocks, types, windows and hints at random, a tenth of the blocks missing in every third problem; the
    same call once more gives the same bits."""
    case = _random(seed)
    print(f"attend random {seed}: {case[:5]} batch {len(case[5])}, {sum(case[5])} new, window {case[7:]}", flush=True)
    p = ah.make(seed, *case, holes=0.1 if seed % 3 == 0 else 0.0)
    got = _attend(p)
    ah.check(p, *got, str(case), ref=_reference64(p))
    again = _attend(p)
    assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1], equal_nan=True)


def test_attend_rows_of_a_projection_on_another_stream():
    """q is a part of wider rows, out as well; the call goes to the stream that is current."""
    from paper_2411_19379_amd import attention as attn
    p = ah.make(4, *LONG["mixed"])
    wide = torch.full((p.T, p.hq + 3, p.d), float("nan"), dtype=p.q.dtype, device=DEV)
    wide[:, 2:2 + p.hq] = p.q.to(DEV)
    out_wide = torch.full_like(wide, 7.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q = wide[:, 2:2 + p.hq] * 1  # made on that stream
        wide[:, 2:2 + p.hq].copy_(q)
        out, lse = attn.attend(wide[:, 2:2 + p.hq], p.k_cache.to(DEV), p.v_cache.to(DEV), _dev(p.table), _dev(p.cu),
                               _dev(np.array(p.cached, np.int32)), scale=p.scale, out=out_wide[:, 1:1 + p.hq], return_lse=True)
    side.synchronize()
    ah.check(p, out.double().cpu().numpy(), lse.cpu().numpy(), ref=_reference64(p))
    assert bool((out_wide[:, 0] == 7.0).all()) and bool((out_wide[:, 1 + p.hq:] == 7.0).all())


def test_attend_offsets_beyond_32_bits():
    """Blocks whose byte offsets in the cache pass 2^32."""
    from paper_2411_19379_amd import attention as attn
    hkv, bs, d = 8, 64, 128
    n_blocks = (5 << 30) // (hkv * bs * d * 2)
    new, cached = [1, 100], [300, 150]
    p = ah.make(6, 16, hkv, d, bs, "bf16", new, cached, max_new=0)
    k = torch.full((n_blocks, hkv, bs, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    v = torch.full_like(k, float("nan"))
    far = {int(b): n_blocks - 1 - i * 3 for i, b in enumerate(sorted(set(p.table[p.table >= 0].tolist())))}
    table = p.table.copy()
    for b, to in far.items():
        k[to], v[to] = p.k_cache[b].to(DEV), p.v_cache[b].to(DEV)
        table[p.table == b] = to
    for max_new in (0, 1):
        out, lse = attn.attend(p.q.to(DEV), k, v, _dev(table), _dev(p.cu), _dev(np.array(cached, np.int32)), scale=p.scale,
                               max_new=max_new, return_lse=True)
        ah.check(p, out.double().cpu().numpy(), lse.cpu().numpy())


@pytest.mark.parametrize("name", sorted(MANY))
def test_attend_many_sequences(name):
    print(f"attend many {name}", flush=True)
    p = many(name)
    ah.check(p, *_attend(p), name)


@pytest.mark.parametrize("name", sorted(PADDED))
def test_attend_rows_of_no_sequence(name):
    print(f"attend padded {name}", flush=True)
    p = padded(name)
    check_padded(p, *_attend(p), name)


def test_attend_a_long_sequence_in_a_step_with_room_for_a_prompt():
    """One token over many keys where the call has rows for a prompt: it is split, and the other rows of `out` stay."""
    from paper_2411_19379_amd import attention as attn
    p = ah.make(8, 8, 2, 128, 16, "bf16", [1], [9000])
    q = torch.zeros((40000, p.hq, p.d), dtype=p.q.dtype, device=DEV)
    q[:1] = p.q.to(DEV)
    out = torch.full_like(q, 7.0)
    _, lse = attn.attend(q, p.k_cache.to(DEV), p.v_cache.to(DEV), _dev(p.table), _dev(p.cu), _dev(np.array(p.cached, np.int32)),
                         scale=p.scale, out=out, return_lse=True)
    ah.check(p, out[:1].double().cpu().numpy(), lse[:1].cpu().numpy(), ref=_reference64(p))
    assert bool((out[1:] == 7.0).all())


def test_attend_widest_window():
    p = ah.make(11, *CASES["chunk_group"])
    ref = ah.reference(p)
    for p.window, p.sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1)):
        ah.check(p, *_attend(p), f"{p.window} {p.sinks}", ref=ref)


@pytest.mark.parametrize("name", ["decode", "decode_group16", "few_tokens", "few_tokens_wide"])
def test_attend_without_the_hint(name):
    """The number of new tokens picks a kernel and nothing else."""
    p = ah.make(11, *CASES[name])
    ref = ah.reference(p)
    for p.max_new in (0, 1, 3, 10 ** 6):
        ah.check(p, *_attend(p), f"{name} {p.max_new}", ref=ref)


def test_nothing_to_do():
    """No sequences, no tokens: empty results, nothing touched."""
    from paper_2411_19379_amd import attention as attn
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    k = torch.ones((4, 2, 16, 64), dtype=torch.bfloat16, device=DEV)
    q, kv = torch.empty((0, 4, 64), dtype=k.dtype, device=DEV), torch.empty((0, 2, 64), dtype=k.dtype, device=DEV)
    for batch in (0, 3):
        s = attn.assign_blocks(16, 0, ints(batch + 1), ints(batch), ints(batch, 5) - 1, ints(8), ints(1) + 8)
        assert s.slots.numel() == 0 and s.positions.numel() == 0 and s.table.shape == (batch, 5) and bool((s.copies[:, :2] == -1).all())
        if batch:
            assert s.counts.tolist() == [8, 0]
        assert attn.rope_append(q, kv, kv, s.positions, s.slots, attn.rotary_table(8, 64), k, k.clone(), copies=s.copies).shape == q.shape
        out, lse = attn.attend(q, k, k, s.table, ints(batch + 1), ints(batch), return_lse=True)
        assert out.shape == q.shape and lse.shape == (0, 4)
    assert bool((k == 1).all())


def _refused():
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device=DEV)
    h = lambda *s: z(*s, t=torch.bfloat16)
    assign = dict(block_size=16, total_tokens=3, cu_seqlens=z(3), cached_lens=z(2), table=z(2, 4), free_blocks=z(8), n_free=z(1))
    rope = dict(q=h(3, 4, 64), k=h(3, 2, 64), v=h(3, 2, 64), positions=z(3), slots=z(3, t=torch.int64) - 1, rotary=z(9, 2, 32, t=torch.float32),
                k_cache=h(5, 2, 16, 64), v_cache=h(5, 2, 16, 64))
    attend = dict(q=h(3, 4, 64), k_cache=h(5, 2, 16, 64), v_cache=h(5, 2, 16, 64), table=z(2, 4), cu_seqlens=z(3), cached_lens=z(2))
    wide = h(3, 2, 4, 64)
    return [
        ("assign_blocks", assign, [
            (dict(cu_seqlens=z(3, t=torch.int64)), ValueError), (dict(cached_lens=z(3)), ValueError), (dict(table=z(4, 4)[::2]), ValueError),
            (dict(n_free=z(2)), ValueError), (dict(shared_tail=z(3)), ValueError), (dict(total_tokens=-1), ValueError),
            (dict(free_blocks=torch.zeros(8, dtype=torch.int32)), ValueError), (dict(block_size=24), RuntimeError), (dict(table=None), TypeError),
            (dict(block_size="16"), TypeError), (dict(block_size=2 ** 40), ValueError), (dict(cu_seqlens=torch.zeros(3, dtype=torch.int32)), ValueError)]),
        ("rope_append", rope, [
            (dict(q=h(3, 4, 64).float()), ValueError), (dict(q=h(4, 4, 64)), ValueError), (dict(k=h(3, 4, 64)), ValueError), (dict(q=wide[:, 0, :, ::2]), ValueError),
            (dict(q=h(3, 64, 4).transpose(1, 2)), ValueError), (dict(slots=z(3)), ValueError),
            (dict(rotary=z(9, 2, 32)), ValueError), (dict(positions=None), TypeError), (dict(k_cache=h(5, 2, 64)), ValueError),
            (dict(v_cache=h(5, 2, 16, 32)), ValueError), (dict(rotary=z(9, 2, 64, t=torch.float32)), RuntimeError), (dict(copies=z(2, 3)), ValueError),
            (dict(q_out=h(3, 4, 32)), ValueError), (dict(q=h(3, 3, 64)), RuntimeError)]),
        ("attend", attend, [
            (dict(q=h(3, 4, 32)), ValueError), (dict(q=h(12, 64)), ValueError), (dict(cu_seqlens=z(4)), ValueError), (dict(table=z(2, 4).long()), ValueError),
            (dict(scale=0.0), RuntimeError), (dict(scale=float("nan")), RuntimeError), (dict(window=-1), RuntimeError), (dict(sinks=-1), RuntimeError),
            (dict(max_new=-1), RuntimeError), (dict(window=2 ** 31), ValueError), (dict(out=h(3, 4, 64).float()), ValueError), (dict(q=h(3, 5, 64)), RuntimeError),
            (dict(k_cache=h(5, 2, 24, 64), v_cache=h(5, 2, 24, 64)), RuntimeError), (dict(q=h(3, 4, 32), k_cache=h(5, 2, 16, 32), v_cache=h(5, 2, 16, 32)), RuntimeError),
            (dict(q=z(3, 4, 64, t=torch.float64)), ValueError), (dict(q=h(3 * 4 * 64 + 1)[1:].view(3, 4, 64)), RuntimeError)]),
    ]


def test_refusals():
    """Wrong types, sizes, strides, devices and values raise before anything is enqueued."""
    from paper_2411_19379_amd import attention as attn
    for name, good, cases in _refused():
        getattr(attn, name)(**good)
        for kw, error in cases:
            with pytest.raises(error):
                getattr(attn, name)(**dict(good, **kw))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", sorted(ASSIGN))
def test_assign(name, in_place):
    from paper_2411_19379_amd import attention as attn
    print(f"assign {name}", flush=True)
    bs, new, cached, forks, n_free = ASSIGN[name]
    rs = np.random.RandomState(1)
    batch, cu = len(new), np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    width = max(-(-(n + c) // bs) for n, c in zip(new, cached)) + 2
    ids = rs.permutation(batch * width + n_free + 3).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    for b, c in enumerate(cached):
        table[b, :-(-c // bs)] = ids[b * width:b * width - (-c // bs)]
    free = np.concatenate([ids[batch * width:batch * width + n_free], [-5, -5]]).astype(np.int32)
    shared = rs.randint(0, 2, batch).astype(np.int32) if forks else None
    want = attn_oracle.assign(bs, cu, cached, table, free, n_free, shared)
    step = attn.assign_blocks(bs, int(cu[-1]), _dev(cu), _dev(np.array(cached, np.int32)), _dev(table), _dev(free),
                              _dev(np.array([n_free], np.int32)), shared_tail=None if shared is None else _dev(shared), in_place=in_place)
    for g, w, what in zip(step, want, ("table", "slots", "positions", "copies", "counts")):
        assert np.array_equal(g.cpu().numpy(), w), f"{name}: {what}"


@pytest.mark.parametrize("name", sorted(ROPE))
def test_rope_append(name):
    from paper_2411_19379_amd import attention as attn
    print(f"rope {name}", flush=True)
    hq, hkv, d, bs, dtype, rot, inter, T = ROPE[name]
    problem = rope_problem(name)
    qkv, caches, rotary, positions, slots, copies = problem
    x, k_cache, v_cache = qkv.to(DEV), caches[0].to(DEV), caches[1].to(DEV)
    q_out = attn.rope_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], _dev(positions), _dev(slots),
                             rotary.to(DEV) if rot else None, k_cache, v_cache, interleaved=bool(inter), copies=_dev(copies))
    rope_check(name, problem, q_out.cpu(), k_cache.cpu(), v_cache.cpu())
    q = x[:, :hq].contiguous()
    same = attn.rope_append(q, x[:, hq:hq + hkv], x[:, hq + hkv:], _dev(positions), _dev(slots),
                            rotary.to(DEV) if rot else None, k_cache, v_cache, interleaved=bool(inter), q_out=q)
    assert same.data_ptr() == q.data_ptr() and torch.equal(q.cpu().view(torch.uint8), q_out.cpu().view(torch.uint8))


def test_a_captured_step_follows_the_lengths():
    """Assign, append and attend captured once and replayed while the lengths on the GPU grow: every replay equals the eager
    calls, with other work and synchronisations between the replays."""
    from paper_2411_19379_amd import attention as attn
    hq, hkv, d, bs, batch = 8, 2, 128, 16, 3
    g = torch.Generator().manual_seed(1)
    n_blocks, width = 64, 16
    cached = torch.tensor([30, 1, 47], dtype=torch.int32, device=DEV)
    cu = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    free = torch.randperm(n_blocks, generator=g).to(torch.int32).to(DEV)
    rotary = attn.rotary_table(width * bs, d)
    qkv = torch.randn((batch, hq + 2 * hkv, d), generator=g).to(torch.bfloat16).to(DEV)

    def start():
        table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        table[0, :2], table[1, :1], table[2, :3] = free[:2], free[2:3], free[3:6]
        gg = torch.Generator().manual_seed(2)
        caches = [torch.randn((n_blocks, hkv, bs, d), generator=gg).to(torch.bfloat16).to(DEV) for _ in range(2)]
        return table, free[6:].contiguous(), torch.tensor([n_blocks - 6], dtype=torch.int32, device=DEV), caches

    def step(x, lens, table, pool, n_free, caches):
        s = attn.assign_blocks(bs, batch, cu, lens, table, pool, n_free, in_place=True)
        q = attn.rope_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], s.positions, s.slots, rotary, *caches)
        out = attn.attend(q, *caches, s.table, cu, lens, max_new=1)
        n_free.copy_(s.counts[:1])
        lens += 1
        return out

    xs = [torch.randn_like(qkv) for _ in range(20)]
    table, pool, n_free, caches = start()
    lens = cached.clone()
    eager = [step(x, lens, table, pool, n_free, caches).clone() for x in xs]

    table, pool, n_free, caches = start()
    lens, x_in = cached.clone(), qkv.clone()
    keep = [t.clone() for t in (table, n_free, *caches, lens)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x_in, lens, table, pool, n_free, caches)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x_in, lens, table, pool, n_free, caches)
    for t, k in zip((table, n_free, *caches, lens), keep):
        t.copy_(k)
    for i, x in enumerate(xs):
        x_in.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]), f"replay {i}"
        attn.attend(xs[0][:, :hq].contiguous(), *caches, table, cu, cached)  # eager work between the replays
    assert lens.tolist() == [50, 21, 67]
