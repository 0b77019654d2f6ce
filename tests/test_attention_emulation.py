"""The attention kernels, compiled for the CPU and run on the SIMT emulator of test_kernel_emulation.py: results against the
definition in 64 bits, every buffer flush against inaccessible pages at its end and at its start, LDS that starts as NaN, and
waves that run in forward, reverse and shuffled order between barriers, which must not change a bit."""
from __future__ import annotations

import os
import subprocess

import numpy as np
import pytest
import torch

import attn_helpers as ah
import attn_oracle
from test_kernel_emulation import CLANG, CSRC, EMU, ROOT, _convert

HERE = os.path.join(ROOT, "tests", "attn_emu")


# Copies from memory into LDS, and the wait for them, which either run at once or (EMU_LATE_COPIES) only when they are waited for:
# the one shows a copy that overwrites what is still read, the other a read in front of the wait.
_LOAD = 'global_load_lds_dwordx4 %0, '
_COPIES = [
    ("    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;",
     "    return (uint32_t)(static_cast<const unsigned char *>(p) - emu::lds_base());"),
    ('    asm volatile("s_mov_b32 m0, %2\\n\\ts_nop 0\\n\\t' + _LOAD + '%1" ::"v"(offset), "s"(from), "s"(to) : "memory");\n',
     "    emu::copy16_to_lds(static_cast<const unsigned char *>(from) + offset, to, __LINE__);\n"),
    ('    asm volatile("s_mov_b32 m0, %1\\n\\ts_nop 0\\n\\t' + _LOAD + 'off" ::"v"(from), "s"(to) : "memory");\n',
     "    emu::copy16_to_lds(from, to, __LINE__);\n"),
    ('    asm volatile("" : "+v"(v));\n', ""),
    ("""asm volatile("s_waitcnt vmcnt(0)" ::: "memory");""", "emu::memory_wait(__LINE__);"),
]


@pytest.fixture(scope="session")
def emu(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ with bf16 vector support found")
    d = str(tmp_path_factory.mktemp("attn_emu"))
    srcs = [os.path.join(EMU, "emu_rt.cpp"), os.path.join(HERE, "emu_attn_main.cpp")]
    for name in ("attn_step", "attn_attend"):
        _convert(os.path.join(CSRC, name + ".hip"), os.path.join(d, name + ".cpp"))
        srcs.append(os.path.join(d, name + ".cpp"))
    common = open(os.path.join(CSRC, "attn_common.h")).read()
    for asm, call in _COPIES:
        assert common.count(asm) == 1, asm
        common = common.replace(asm, call)
    open(os.path.join(d, "common.h"), "w").write(common)
    _convert(os.path.join(d, "common.h"), os.path.join(d, "attn_common.h"))
    flags = ["-std=c++17", "-O2", "-fno-strict-aliasing", "-ffp-contract=off", "-Wno-psabi", "-Wno-unused-value",
             "-DATTN_TARGET=emu::env_int(\"EMU_TARGET\")", "-I", d, "-I", HERE, "-I", EMU, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    procs = [subprocess.Popen([CLANG, *flags, "-c", s, "-o", os.path.join(d, f"{i}.o")], stderr=subprocess.PIPE, text=True)
             for i, s in enumerate(srcs)]
    for p in procs:
        _, err = p.communicate()
        assert p.returncode == 0, err[-3000:]
    exe = os.path.join(d, "emu_attn_main")
    subprocess.run([CLANG, *[os.path.join(d, f"{i}.o") for i in range(len(srcs))], "-o", exe], check=True)
    return exe


def _bits(t):
    """A tensor's bytes."""
    t = t.contiguous()
    return (t.view(torch.int32) if t.dtype == torch.float32 else t.view(torch.int16)).numpy().tobytes()


def _run(exe, tmp_path, op, params, arrays, order=0, side="end", target=0, late=0):
    src, dst = str(tmp_path / "in.bin"), str(tmp_path / "out.bin")
    words = np.zeros(34, np.int32)
    words[0], words[1] = 0x4154544e, op
    words[2:2 + len(params)] = params
    with open(src, "wb") as f:
        f.write(words.tobytes())
        for a in arrays:
            f.write(a if isinstance(a, bytes) else np.ascontiguousarray(a).tobytes())
    env = dict(os.environ, EMU_TARGET=str(target), EMU_LATE_COPIES=str(late))
    r = subprocess.run([exe, src, dst, str(order), side], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])
    return open(dst, "rb").read()


def _attend(exe, tmp_path, p, order=0, side="end", target=0, gap=0, late=0):
    """`gap`: elements between the tokens of q beyond their heads."""
    row = p.hq * p.d
    q = torch.full((p.T, row + gap), float("nan"), dtype=p.q.dtype)
    q[:, :row] = p.q.reshape(p.T, row)
    flat = q.reshape(-1)[:max(0, p.T * (row + gap) - gap)]
    params = [p.hq, p.hkv, p.d, p.bs, ah.CODE[p.dtype], p.T, len(p.new), p.k_cache.shape[0], p.table.shape[1], p.window, p.sinks,
              p.max_new, int(np.float32(p.scale).view(np.int32)), row + gap]
    raw = _run(exe, tmp_path, 2, params, [_bits(flat), _bits(p.k_cache), _bits(p.v_cache), p.table, p.cu, np.array(p.cached, np.int32)],
               order, side, target, late)
    esz = p.q.element_size()
    n = p.T * row
    out = torch.frombuffer(bytearray(raw[:n * esz]) or bytearray(esz), dtype=p.q.dtype)[:n].double().numpy().reshape(p.T, p.hq, p.d)
    return out, np.frombuffer(raw[n * esz:], np.float32).reshape(p.T, p.hq)


# heads, key heads, head_dim, block size, type, new tokens, cached tokens, window, sinks, max_new
CASES = {
    "one_token": (4, 1, 128, 16, "bf16", [1], [0], 0, 0, 1),
    "decode": (8, 2, 64, 8, "f16", [1, 1, 0, 1], [37, 200, 9, 63], 0, 0, 1),
    "decode_group16": (16, 1, 128, 32, "bf16", [1, 1], [130, 31], 0, 0, 1),
    "decode_group24": (24, 1, 64, 16, "bf16", [1], [70], 0, 0, 1),
    "few_tokens": (4, 2, 128, 16, "f16", [5, 2, 1], [40, 0, 77], 0, 0, 5),
    "few_tokens_wide": (12, 1, 64, 16, "bf16", [5], [40], 0, 0, 5),
    "few_window": (3, 3, 64, 4, "bf16", [1, 7], [150, 97], 20, 3, 7),
    "few_by_a_wrong_hint": (2, 1, 64, 16, "f16", [40, 3], [5, 30], 0, 0, 1),
    "chunk": (2, 2, 64, 16, "bf16", [70], [33], 0, 0, 0),
    "chunk_group": (4, 1, 128, 16, "f16", [67, 1, 0, 20], [10, 80, 5, 0], 0, 0, 0),
    "chunk_group3": (3, 1, 64, 1, "bf16", [100], [0], 0, 0, 0),
    "chunk_window": (2, 1, 64, 32, "bf16", [150], [100], 70, 5, 0),
    "chunk_window1": (2, 2, 64, 16, "f16", [65, 3], [70, 64], 1, 0, 0),
    "chunk_many_sinks": (4, 4, 64, 16, "bf16", [66], [140], 10, 70, 0),
    "f32": (4, 2, 64, 16, "f32", [37, 1], [20, 64], 0, 0, 0),
    "f32_wide_window": (2, 1, 128, 8, "f32", [40, 0, 2], [61, 7, 33], 17, 2, 0),
}


@pytest.mark.parametrize("name,target", [(name, 60) for name in sorted(CASES)] + [(name, 2) for name in sorted(CASES)] +
                         [(name, 0) for name in ("chunk_group", "decode", "f32", "few_tokens", "few_tokens_wide")])
def test_attend(emu, tmp_path, name, target):
    p = ah.make(11, *CASES[name])
    out, lse = _attend(emu, tmp_path, p, target=target)
    ah.check(p, out, lse, name)
    # (most of the workgroups of target 0, the one that is used, have nothing to do)
    for order, side, late in ((1, "start", 1), (5, "end", 0), (4, "end", 1)) if target else ((5, "start", 1),):
        other = _attend(emu, tmp_path, p, order, side, target, late=late)
        assert np.array_equal(out, other[0]) and np.array_equal(lse, other[1]), f"{name}: order {order} changes the result"


@pytest.mark.parametrize("name", ["decode", "few_window", "chunk", "chunk_window", "f32_wide_window"])
def test_attend_with_blocks_missing(emu, tmp_path, name):
    """Table entries that name no block: their keys are not seen, and rows that see nothing come out as zeros."""
    case = CASES[name]
    p = ah.make(5, *case, holes=0.5)
    if name == "decode":
        p.table[0] = -1
    for target in (2, 40):
        out, lse = _attend(emu, tmp_path, p, target=target, gap=16)
        ah.check(p, out, lse, name)
    if name == "decode":
        assert np.all(out[0] == 0) and np.all(np.isneginf(lse[0]))


@pytest.mark.parametrize("name", ["decode", "few_window", "chunk", "f32"])
def test_attend_with_a_table_that_is_too_narrow(emu, tmp_path, name):
    """Sequences longer than their rows of the table: the keys behind its end do not exist."""
    p = ah.make(13, *CASES[name])
    for width in (1, 3):
        p.table = np.ascontiguousarray(ah.make(13, *CASES[name]).table[:, :width])
        for target in (2, 40):
            out, lse = _attend(emu, tmp_path, p, target=target)
            ah.check(p, out, lse, f"{name} {width}")


NOT_FINITE = ["few_window", "few_tokens", "chunk_window", "chunk_group", "f32_wide_window"]


@pytest.mark.parametrize("where", ["v", "k"])
@pytest.mark.parametrize("name", NOT_FINITE)
def test_attend_not_finite_stays_with_the_rows_that_see_it(emu, tmp_path, name, where):
    """Infinities and NaN in keys and values, of cached and of new tokens."""
    p = ah.make(7, *CASES[name])
    cache = p.v_cache if where == "v" else p.k_cache
    for i, bad in enumerate([float("inf"), float("nan"), -float("inf")]):
        seq = max(range(len(p.new)), key=lambda b: p.new[b])
        total = p.new[seq] + p.cached[seq]
        for j in {total - 1 - 2 * i, total // 2 + i, total * 3 // 4 - i}:
            if 0 <= j < total:
                block, row = p.block_row(seq, j)
                cache[block, i % p.hkv, row, (5 * i + j) % p.d] = bad
    for target in (2, 30):
        out, lse = _attend(emu, tmp_path, p, target=target)
        ah.check(p, out, lse, name)


def test_attend_scores_of_minus_infinity_alone(emu, tmp_path):
    """All scores minus infinity: the softmax is undefined, unlike that of a row that sees nothing; a finite one decides."""
    for dtype, d in (("bf16", 64), ("f32", 64)):
        p = ah.make(3, 1, 1, d, 16, dtype, [1, 70, 1], [40, 40, 40], max_new=0)
        p.q[:] = torch.abs(p.q)
        for b in (0, 2):
            for j in range(41):
                if b == 0 or j != 20:
                    block, row = p.block_row(b, j)
                    p.k_cache[block, 0, row] = -float("inf")
        for max_new in (0, 1):
            p.max_new = max_new
            for target in (2, 9):
                out, lse = _attend(emu, tmp_path, p, target=target)
                assert np.isnan(out[0]).all() and np.isfinite(out[71]).all()
                ah.check(p, out, lse, f"{dtype} {max_new} {target}")


def test_attend_large_scores(emu, tmp_path):
    """Scores that grow along the keys far beyond what exp holds."""
    for dtype in ("bf16", "f16", "f32"):
        for max_new in (1, 0):
            p = ah.make(9, 2, 1, 64, 16, dtype, [1, 66], [200, 90], max_new=max_new, spread=1.0)
            for b in range(2):
                for j in range(p.new[b] + p.cached[b]):
                    block, row = p.block_row(b, j)
                    p.k_cache[block, 0, row, 0] = 0.5 * j
            p.q[:, :, 0] = 40.0
            out, lse = _attend(emu, tmp_path, p, target=20)
            ah.check(p, out, lse, dtype, sums=0.0 if dtype != "f32" else 40.0 * 0.5 * 200 * p.scale)


# More sequences than a wave looks up at once, and than it looks up four to a lane.
MANY = {
    "few_70": (2, 1, 64, 16, "bf16", [1] * 70, [(37 * i) % 150 for i in range(70)], 0, 0, 1),
    "few_300": (1, 1, 64, 8, "f16", [i % 7 != 3 for i in range(300)], [(5 * i) % 41 for i in range(299)] + [170], 0, 0, 1),
    "few_300_window": (2, 2, 64, 8, "f16", [i % 3 for i in range(300)], [(5 * i) % 41 for i in range(299)] + [170], 9, 2, 2),
    "chunk_70": (2, 1, 64, 16, "bf16", [i % 4 for i in range(68)] + [70, 3], [(11 * i) % 60 for i in range(69)] + [300], 0, 0, 0),
    "chunk_300": (1, 1, 64, 16, "f16", [40] + [i % 2 for i in range(298)] + [60], [0] + [i % 19 for i in range(298)] + [130], 0, 0, 60),
    "f32_300": (1, 1, 64, 16, "f32", [i % 2 for i in range(299)] + [40], [i % 19 for i in range(299)] + [70], 0, 0, 0),
}


def many(name):
    hq, hkv, d, bs, dtype, new, *rest = MANY[name]
    return ah.make(17, hq, hkv, d, bs, dtype, [int(n) for n in new], *rest)


@pytest.mark.parametrize("name", sorted(MANY))
def test_attend_many_sequences(emu, tmp_path, name):
    p = many(name)
    ah.check(p, *_attend(emu, tmp_path, p, target=400), name)


# heads, key heads, head_dim, block size, type, new tokens (the last ones belong to no sequence), cached tokens
PADDED = {
    "chunk": (2, 1, 64, 16, "bf16", [10, 600], [300, 0], 0, 0, 0),
    "chunk_three": (2, 1, 64, 16, "f16", [70, 0, 3, 200], [300, 5, 40, 0], 0, 0, 0),
    "few": (4, 2, 128, 16, "bf16", [1, 1, 30], [260, 40, 0], 0, 0, 1),
    "f32": (2, 1, 64, 16, "f32", [3, 130], [150, 0], 0, 0, 0),
    "nothing": (2, 1, 64, 16, "bf16", [0, 90], [150, 0], 0, 0, 0),
}


class Padded(ah.Problem):
    """A problem with more rows than its sequences have tokens."""

    @property
    def T(self):
        return int(self.q.shape[0])


def padded(name):
    p = ah.make(19, *PADDED[name])
    return Padded(**dict(vars(p), new=p.new[:-1], cached=p.cached[:-1], table=np.ascontiguousarray(p.table[:-1]), cu=p.cu[:-1]))


def check_padded(p, out, lse, what):
    n = int(p.cu[-1])
    ah.check(p, out[:n], lse[:n], what, ref=[x[:n] for x in ah.reference(p)])


@pytest.mark.parametrize("target", [2, 30])
@pytest.mark.parametrize("name", sorted(PADDED))
def test_attend_rows_of_no_sequence(emu, tmp_path, name, target):
    """cu_seqlens ends in front of the rows' end, as in a captured step with room for more tokens; a single sequence that has few
    of them and many keys is split all the same."""
    p = padded(name)
    check_padded(p, *_attend(emu, tmp_path, p, target=target), name)


@pytest.mark.parametrize("name", ["chunk", "few"])
def test_attend_widest_window(emu, tmp_path, name):
    """Windows and sinks up to the type's largest see what no window sees."""
    p = ah.make(11, *CASES["chunk_group" if name == "chunk" else "few_tokens"])
    ref = ah.reference(p)
    for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1)):
        p.window, p.sinks = window, sinks
        for target in (2, 40):
            ah.check(p, *_attend(emu, tmp_path, p, target=target), f"{name} {window} {sinks}", ref=ref)


ASSIGN = {
    "one": (16, [137], [1001], True, 64),
    "mixed": (8, [1, 0, 30, 8, 5, 0, 17], [0, 12, 7, 8, 9, 8, 1], True, 40),
    "tokens": (1, [3, 1, 4], [2, 0, 6], True, 20),
    "short": (4, [9, 9, 9, 0, 2], [3, 4, 6, 2, 1], True, 5),
    "none_free": (4, [3, 2], [6, 8], True, 0),
    "no_tokens": (4, [0, 0], [6, 8], True, 3),
    "many": (2, [1 + i % 5 for i in range(300)], [i % 9 for i in range(300)], False, 2000),
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", sorted(ASSIGN))
def test_assign(emu, tmp_path, name, in_place):
    bs, new, cached, forks, n_free = ASSIGN[name]
    rs = np.random.RandomState(1)
    batch, cu = len(new), np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    width = max(-(-(n + c) // bs) for n, c in zip(new, cached)) + 2
    ids = rs.permutation(batch * width + n_free + 3).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    for b, c in enumerate(cached):
        table[b, :-(-c // bs)] = ids[b * width:b * width - (-c // bs)]
    free = np.concatenate([ids[batch * width:batch * width + n_free], [-5, -5]]).astype(np.int32)  # more room than free blocks
    shared = rs.randint(0, 2, batch).astype(np.int32) if forks else None
    want = attn_oracle.assign(bs, cu, cached, table, free, n_free, shared)
    T = int(cu[-1])
    for order, side in ((0, "end"), (1, "start"), (4, "end")):
        raw = _run(emu, tmp_path, 0, [batch, bs.bit_length() - 1, width, T, shared is not None, len(free), in_place],
                   [cu, np.array(cached, np.int32), *([shared] if shared is not None else []), table, free, np.array([n_free], np.int32)], order, side)
        sizes, got = [(np.int32, batch * width), (np.int64, T), (np.int32, T), (np.int32, batch * 4), (np.int32, 2)], []
        for t, n in sizes:
            got.append(np.frombuffer(raw[:n * t().itemsize], t))
            raw = raw[n * t().itemsize:]
        for g, w, what in zip(got, want, ("table", "slots", "positions", "copies", "counts")):
            assert np.array_equal(g, w.reshape(-1)), f"{name}: {what}"


# heads, key heads, head_dim, block size, type, rotary_dim, interleaved, tokens
ROPE = {
    "half": (4, 2, 128, 16, "bf16", 128, 0, 9),
    "part": (3, 3, 64, 8, "f16", 32, 0, 5),
    "interleaved": (2, 1, 64, 4, "f32", 64, 1, 7),
    "interleaved_part": (5, 1, 256, 16, "bf16", 16, 1, 3),
    "odd_head": (2, 2, 24, 2, "f32", 16, 0, 4),
    "none": (2, 1, 64, 4, "f16", 0, 0, 6),
}


def rope_tolerance(dtype, size):
    """Two products and a sum in fp32, at most 3 half ulps of the pair's length, and one rounding to the type."""
    u = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    return (u + 3 * 2.0 ** -24) * size + (2.0 ** -25 if dtype == "f16" else 1e-37)


def rope_problem(name, seed=2):
    hq, hkv, d, bs, dtype, rot, inter, T = ROPE[name]
    g = torch.Generator().manual_seed(seed)
    rs = np.random.RandomState(seed)
    t = ah.TORCH[dtype]
    n_blocks, most = T + 3, 50
    qkv = torch.randn((T, hq + 2 * hkv, d), generator=g).to(t)
    caches = [torch.randn((n_blocks, hkv, bs, d), generator=g).to(t) for _ in range(2)]
    rotary = torch.randn((most, 2, max(rot // 2, 1)), generator=g)[:, :, :rot // 2].contiguous()
    positions = rs.randint(0, most, T).astype(np.int32)
    slots = rs.permutation((n_blocks - 2) * bs)[:T].astype(np.int64)
    slots[1] = -1                   # a token that got no block
    slots[2] = n_blocks * bs + 5    # and one whose block is not of this cache
    positions[0] = most             # a position behind the table
    copies = np.array([[n_blocks - 2, n_blocks - 1, bs - 1, 0], [-1, -1, 0, 0], [n_blocks - 2, -1, 1, 0]], np.int32)
    return qkv, caches, rotary, positions, slots, copies


def rope_check(name, problem, q_out, k_cache, v_cache):
    hq, hkv, d, bs, dtype, rot, inter, T = ROPE[name]
    qkv, caches, rotary, positions, slots, copies = problem
    rows = rotary.numpy()[np.minimum(positions, rotary.shape[0] - 1)].copy()
    x = qkv.double().numpy()
    if rot:
        rows[positions >= rotary.shape[0]] = np.nan
    y = attn_oracle.turn(x[:, :hq + hkv], rows, rot, inter)
    size = np.abs(x[:, :hq + hkv]).max() * 2 * max(1.0, float(rotary.abs().max()) if rot else 1.0)
    tol = rope_tolerance(dtype, size)
    def close(got, want, what):
        assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in {what}"
        assert np.nanmax(np.abs(got - want), initial=0.0) <= tol, f"{name}: {what}"
        if rot < d:
            assert np.array_equal(got[..., rot:], want[..., rot:]), f"{name}: the part of {what} that does not turn"
    close(q_out.double().numpy(), y[:, :hq], "q")
    n_blocks = caches[0].shape[0]
    want_k, want_v = (c.double().numpy().copy() for c in caches)
    for w in (want_k, want_v):
        src, dst, n, _ = copies[0]
        w[dst, :, :n] = w[src, :, :n]
    for t in range(T):
        if 0 <= slots[t] < n_blocks * bs:
            want_k[slots[t] // bs, :, slots[t] % bs] = y[t, hq:]
            want_v[slots[t] // bs, :, slots[t] % bs] = x[t, hq + hkv:]
    close(k_cache.double().numpy(), want_k, "the keys")
    assert np.array_equal(v_cache.double().numpy(), want_v), f"{name}: the values"


@pytest.mark.parametrize("name", sorted(ROPE))
def test_rope_append(emu, tmp_path, name):
    hq, hkv, d, bs, dtype, rot, inter, T = ROPE[name]
    problem = rope_problem(name)
    qkv, caches, rotary, positions, slots, copies = problem
    for order, side in ((0, "end"), (1, "start")):
        raw = _run(emu, tmp_path, 1, [hq, hkv, d, bs, ah.CODE[dtype], T, 3, caches[0].shape[0], rotary.shape[0], rot, inter, 1, (hq + 2 * hkv) * d],
                   [_bits(qkv), positions, slots, rotary.numpy(), copies, _bits(caches[0]), _bits(caches[1])], order, side)
        t, esz = qkv.dtype, qkv.element_size()
        nq, nc = T * hq * d, caches[0].numel()
        flat = torch.frombuffer(bytearray(raw), dtype=t)
        rope_check(name, problem, flat[:nq].view(T, hq, d), flat[nq:nq + nc].view(caches[0].shape), flat[nq + nc:].view(caches[0].shape))
