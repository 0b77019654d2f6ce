"""Arguments at the edge of what the entry points take, and index arrays that no caller should pass: lengths that decrease, are
negative or reach behind the arrays, sequences that name the same tokens, blocks and positions of nowhere.  Every buffer of the
emulation lies against inaccessible pages, so an access outside the arguments ends the run; what the operators say of such a
call has to make sense all the same."""
import numpy as np
import pytest
import torch

import attn_helpers as ah
from test_attention_emulation import CASES, _attend, _run, emu  # noqa: F401

MOST = 2 ** 31 - 1


def _assign(exe, tmp_path, bs, T, cu, cached, table, free, n_free, shared=None, in_place=False, **kw):
    cu, cached, table, free = (np.array(x, np.int32) for x in (cu, cached, table, free))
    batch, width = table.shape
    raw = _run(exe, tmp_path, 0, [batch, bs.bit_length() - 1, width, T, shared is not None, len(free), in_place],
               [cu, cached, *([np.array(shared, np.int32)] if shared is not None else []), table, free, np.array([n_free], np.int32)], **kw)
    got = []
    for t, shape in ((np.int32, (batch, width)), (np.int64, T), (np.int32, T), (np.int32, (batch, 4)), (np.int32, 2)):
        n = int(np.prod(shape)) * t().itemsize
        got.append(np.frombuffer(raw[:n], t).reshape(shape))
        raw = raw[n:]
    return got


def test_assign_needs_beyond_32_bits(emu, tmp_path):
    """2048 sequences that all name the same tokens: their needs add up to more than 2^31."""
    batch, T, free = 4096, 2 ** 20 + 4096, np.arange(100, 116)
    cu = np.array([0 if b % 2 == 0 else T for b in range(batch + 1)])
    table, slots, positions, copies, counts = _assign(emu, tmp_path, 1, T, cu, np.zeros(batch), np.full((batch, 2), -1), free, 16)
    assert counts.tolist() == [0, MOST]
    assert set(np.unique(table)) <= {-1, *free} and set(np.unique(slots)) <= {-1, *free}
    given = table[table >= 0]
    assert len(set(given)) == len(given) and np.all(copies[:, :2] == -1)


# Tables whose rows end in front of the last token: block size, width, new, cached, free blocks.
NARROW = {
    "some": (4, 2, [20], [2], 10),
    "behind": (4, 2, [5], [11], 10),
    "last_entry": (4, 2, [3, 1], [5, 8], 10),
    "several": (8, 3, [1, 0, 30, 8, 5, 0, 17, 2], [0, 40, 7, 24, 23, 8, 30, 16], 40),
    "and_short": (8, 3, [1, 0, 30, 8, 5, 0, 17, 2], [0, 40, 7, 24, 23, 8, 30, 16], 3),
    "tokens": (1, 1, [3, 1, 4], [2, 0, 0], 20),
    "many": (2, 2, [1 + i % 5 for i in range(300)], [i % 9 for i in range(300)], 350),
}


def narrow_problem(name):
    """The call's arrays and what it has to say: entries behind the row's end take no block, and count as missing where new
    tokens are theirs."""
    bs, width, new, cached, n_free = NARROW[name]
    batch = len(new)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    for b, c in enumerate(cached):
        held = min(-(-c // bs), width)
        table[b, :held] = b * width + np.arange(held)
    free = 10000 + np.arange(n_free, dtype=np.int32)
    shared = (np.arange(batch) % 3 != 1).astype(np.int32)
    out, left, missing, slots, positions, copies = table.copy(), n_free, 0, [], [], []
    for b, (n, c) in enumerate(zip(new, cached)):
        copies.append([-1, -1, 0, 0])
        for e in range(c // bs, -(-(c + n) // bs) if n else 0):
            old = e < -(-c // bs)
            if old and not shared[b] and e < width:
                continue  # the last cached block takes more tokens
            if e >= width or left == 0:
                block, missing = -1, missing + 1
            else:
                left -= 1
                block = int(free[left])
            if e < width:
                if old:
                    copies[-1] = [int(table[b, e]), block, c % bs, 0]
                out[b, e] = block
        for p in range(c, c + n):
            block = int(out[b, p // bs]) if p // bs < width else -1
            slots.append(block * bs + p % bs if block >= 0 else -1)
            positions.append(p)
    want = (out, np.array(slots, np.int64), np.array(positions, np.int32), np.array(copies, np.int32), np.array([left, missing], np.int32))
    return (bs, int(cu[-1]), cu, np.array(cached, np.int32), table, free, n_free, shared), want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", sorted(NARROW))
def test_assign_with_a_table_that_is_too_narrow(emu, tmp_path, name, in_place):
    args, want = narrow_problem(name)
    for order, side in ((0, "end"), (1, "start")):
        got = _assign(emu, tmp_path, *args, in_place=in_place, order=order, side=side)
        for g, w, what in zip(got, want, ("table", "slots", "positions", "copies", "counts")):
            assert np.array_equal(g, w), f"{name}: {what}"


# cu_seqlens, cached_lens; 40 tokens
LENGTHS = {
    "decreasing": ([0, 30, 10, 40], [5, 0, 9]),
    "negative": ([-7, -3, 12, 40], [-5, 3, -2 ** 31]),
    "behind_the_end": ([0, 50, 1000, MOST], [5, 4, 3]),
    "far_behind": ([MOST, MOST, 0, 40], [MOST, MOST, MOST]),
    "late_start": ([9, 9, 20, 38], [1, 2, 3]),
    "long_cached": ([0, 10, 20, 40], [MOST, 2 ** 30, 100000]),
    "all_the_same": ([0, 40, 0, 40], [0, 17, 2]),
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", sorted(LENGTHS))
def test_assign_lengths(emu, tmp_path, name, in_place):
    cu, cached = LENGTHS[name]
    held, free = np.arange(18).reshape(3, 6), np.arange(100, 120)
    for bs in (1, 8):
        for n_free in (-3, 0, 11, 20, MOST):
            table, slots, positions, copies, counts = _assign(emu, tmp_path, bs, 40, cu, cached, held, free, n_free, shared=[1, 0, -1],
                                                              in_place=in_place, side="end" if bs == 1 else "start")
            most = min(max(n_free, 0), 20)
            assert 0 <= counts[0] <= most and counts[1] >= 0
            assert set(np.unique(table)) <= {-1, *held.ravel(), *free}
            blocks = slots[slots >= 0] // bs
            assert set(np.unique(blocks)) <= {*held.ravel(), *free} and np.all(slots >= -1) and np.all(positions >= 0)
            given = table[table >= 100]
            assert len(set(given)) == len(given) <= most - counts[0]


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("case", ["few_window", "chunk_group", "f32"])
def test_attend_lengths(emu, tmp_path, case, name):
    """Rows of the arguments alone are written, and read keys come from the cache: a row's results are means of its values."""
    hq, hkv, d, bs, dtype, _, _, window, sinks, max_new = {
        "few_window": (3, 3, 64, 4, "bf16", 0, 0, 20, 3, 1), "chunk_group": (4, 1, 64, 16, "f16", 0, 0, 0, 0, 0),
        "f32": (4, 2, 64, 16, "f32", 0, 0, 0, 0, 0)}[case]
    p = ah.make(3, hq, hkv, d, bs, dtype, [10, 20, 10], [30, 20, 40], window, sinks, max_new, spare=0)
    p.k_cache[:] = p.k_cache.nan_to_num(0.0)
    p.v_cache[:] = p.v_cache.nan_to_num(0.0)
    most = float(p.v_cache.abs().max()) * (1 + 2.0 ** -7)
    cu, p.cached = np.array(LENGTHS[name][0], np.int32), LENGTHS[name][1]
    T = p.T
    p.cu = cu
    p.__class__ = type("Cut", (ah.Problem,), {"T": property(lambda self: T)})
    for target, side in ((2, "end"), (30, "start")):
        out, lse = _attend(emu, tmp_path, p, target=target, side=side)
        # rows of no sequence keep the NaN patterns they started with
        assert np.all(np.isnan(out) | (np.abs(out) <= most))
        assert not np.any(np.isposinf(lse))


def test_append_nowhere(emu, tmp_path):
    """Slots, positions and copies of nowhere: only what lies in the caches is written."""
    hq, hkv, d, bs, T, n_blocks, most = 2, 1, 64, 4, 9, 3, 5
    rs = np.random.RandomState(1)
    qkv, rotary = rs.randn(T, (hq + 2 * hkv) * d).astype(np.float32), rs.randn(most, 2, 16).astype(np.float32)
    caches = [rs.randn(n_blocks, hkv, bs, d).astype(np.float32) for _ in "kv"]
    positions = np.array([-1, 5, MOST, -2 ** 31, 0, 1, 2, 3, 4], np.int32)
    slots = np.array([-1, 12, 2 ** 40, -2 ** 63, 2 ** 63 - 1, 2 ** 32, 11, -2 ** 32, 0], np.int64)
    copies = np.array([[0, 3, 4, 0], [-1, 2, 4, 0], [2 ** 31 - 1, 1, 4, 0], [1, -2 ** 31, 4, 0], [1, 2, -9, 0]], np.int32)
    raw = _run(emu, tmp_path, 1, [hq, hkv, d, bs, 0, T, len(copies), n_blocks, most, 32, 0, 1, (hq + 2 * hkv) * d],
               [qkv, positions, slots, rotary, copies, *caches])
    flat = np.frombuffer(raw, np.float32)
    k, v = flat[T * hq * d:].reshape(2, n_blocks, hkv, bs, d)
    kept = np.ones((n_blocks, bs), bool)
    kept[2, 3] = kept[0, 0] = False
    for got, was, part in ((k, caches[0], 2), (v, caches[1], 3)):
        assert np.array_equal(got[:, 0][kept], was[:, 0][kept])
        assert np.array_equal(got[2, 0, 3, 32:], qkv[6].reshape(-1, d)[part, 32:]) and np.array_equal(got[0, 0, 0, 32:], qkv[8].reshape(-1, d)[part, 32:])
    q = flat[:T * hq * d].reshape(T, hq, d)
    assert np.isnan(q[:4, :, :32]).all() and np.isfinite(q[4:]).all()


@pytest.mark.parametrize("scale", [8.3e-39, 1.3e-38, 2.3e-38, 2.4e-38])
@pytest.mark.parametrize("name", ["decode", "few_tokens_wide", "chunk", "f32"])
def test_attend_smallest_scales(emu, tmp_path, name, scale):
    """From the smallest scale that is accepted on: every key weighs the same, and lse is the log of their number."""
    p = ah.make(11, *CASES[name])
    p.scale = float(np.float32(scale))
    for target in (2, 30):
        ah.check(p, *_attend(emu, tmp_path, p, target=target), f"{name} {scale}")


@pytest.mark.parametrize("name", ["decode", "few_tokens_wide", "chunk_group", "f32"])
def test_attend_scores_beyond_fp32(emu, tmp_path, name):
    """A row whose largest scaled score has no place in fp32 says so: NaN, not the zeros of a row that sees nothing."""
    p = ah.make(11, *CASES[name])
    p.scale = 1e38
    top = np.full((p.T, p.hq), np.nan)
    for b, (n, c) in enumerate(zip(p.new, p.cached)):
        for i in range(n):
            rows = [p.block_row(b, j) for j in range(c + i + 1)]
            for h in range(p.hq):
                k = np.stack([p.k_cache[block, h // (p.hq // p.hkv), r].double().numpy() for block, r in rows])
                top[p.cu[b] + i, h] = (k @ p.q[p.cu[b] + i, h].double().numpy()).max()
    beyond = np.abs(top) > 4.0  # 4e38 is behind fp32's end
    assert beyond.sum() > 0.5 * beyond.size
    for target in (2, 30):
        out, lse = _attend(emu, tmp_path, p, target=target)
        assert np.isnan(out[beyond]).all() and np.isnan(lse[beyond]).all(), f"{name} {target}"


def light_weights(max_new, dtype="f16", keys=1500, new=1):
    """One key in front outweighs each of the others by 2^24 to 2^28; its value is 0, theirs are around 1000."""
    p = ah.make(29, 2, 1, 64, 16, dtype, [new], [keys], max_new=max_new)
    g = torch.Generator().manual_seed(4)
    p.q[:] = 0
    p.q[:, :, 0] = 8.0
    for j in range(keys + new):
        block, row = p.block_row(0, j)
        p.k_cache[block, 0, row] = 0
        p.k_cache[block, 0, row, 0] = 18.0 if j == 0 else float(torch.rand(1, generator=g)) * 2.8 - 1.4
        p.v_cache[block, 0, row] = 0 if j == 0 else (1000 + 50 * torch.randn(64, generator=g)).to(p.v_cache.dtype)
    return p


def check_light_weights(p, out, lse, what):
    """A weight of fp16 is off by half an ulp or, below the smallest normal number, by 2^-25; the largest of a row is 2^7 at least.
    The result is rounded once, and its own subnormal numbers are 2^-24 apart."""
    want, want_lse, size = ah.reference(p)
    u = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[p.dtype]
    tol = (2 * u + 1e-5) * size + ((p.new[0] + p.cached[0]) * 1200 * 2.0 ** -32 + 2.0 ** -25 if p.dtype == "f16" else 0)
    assert np.all(tol < 0.1 * np.abs(want))  # a row without them is far out
    assert np.abs(out - want).max() <= tol.max() and np.all(np.abs(out - want) <= tol), f"{what}: {(np.abs(out - want) / tol).max():.1f} times the bound"
    assert np.all(np.abs(lse - want_lse) <= 1e-5 * (1 + np.abs(want_lse)))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("max_new,new", [(1, 1), (0, 40)])
def test_attend_many_light_keys(emu, tmp_path, max_new, new, dtype):
    """Weights far below a row's largest one count, in the sum with v as in the sum of weights."""
    p = light_weights(max_new, dtype, new=new)
    for target in (1, 20):
        check_light_weights(p, *_attend(emu, tmp_path, p, target=target), f"{new} {target}")
