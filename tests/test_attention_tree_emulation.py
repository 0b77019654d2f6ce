"""The kernels of steps that check trees of drafted tokens on the SIMT emulator: against the definition in 64 bits, with every buffer
flush against inaccessible pages and the waves in several orders, which must not change a bit."""
from __future__ import annotations

import os
import subprocess

import numpy as np
import pytest
import torch

import attn_helpers as ah
import tree_helpers as th
import tree_oracle
from test_attention_emulation import _COPIES, _bits, _run
from test_kernel_emulation import CLANG, CSRC, EMU, ROOT, _convert

HERE = os.path.join(ROOT, "tests", "attn_emu")


@pytest.fixture(scope="session")
def emu(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ with bf16 vector support found")
    d = str(tmp_path_factory.mktemp("tree_emu"))
    srcs = [os.path.join(EMU, "emu_rt.cpp"), os.path.join(HERE, "emu_tree_main.cpp")]
    waits = 'asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");'
    for name in ("attn_tree", "attn_attend", "attn_tree_attend"):
        source = open(os.path.join(CSRC, name + ".hip")).read()
        assert source.count(waits) == (name == "attn_tree_attend")
        open(os.path.join(d, name + ".hip"), "w").write(source.replace(waits, "emu::memory_wait_but(N, __LINE__);"))
        _convert(os.path.join(d, name + ".hip"), os.path.join(d, name + ".cpp"))
        srcs.append(os.path.join(d, name + ".cpp"))
    common = open(os.path.join(CSRC, "attn_common.h")).read()
    for asm, call in _COPIES:
        assert common.count(asm) == 1, asm
        common = common.replace(asm, call)
    open(os.path.join(d, "common.h"), "w").write(common)
    _convert(os.path.join(d, "common.h"), os.path.join(d, "attn_common.h"))
    flags = ["-std=c++17", "-O2", "-fno-strict-aliasing", "-ffp-contract=off", "-Wno-psabi", "-Wno-unused-value", "-D__popcll=__builtin_popcountll",
             "-include", os.path.join(HERE, "tree_emu.h"), "-DATTN_TARGET=emu::env_int(\"EMU_TARGET\")", "-I", d, "-I", HERE, "-I", EMU, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    procs = [subprocess.Popen([CLANG, *flags, "-c", s, "-o", os.path.join(d, f"{i}.o")], stderr=subprocess.PIPE, text=True)
             for i, s in enumerate(srcs)]
    for p in procs:
        _, err = p.communicate()
        assert p.returncode == 0, err[-3000:]
    exe = os.path.join(d, "emu_tree_main")
    subprocess.run([CLANG, *[os.path.join(d, f"{i}.o") for i in range(len(srcs))], "-o", exe], check=True)
    return exe


ORDERS = [(0, "end"), (1, "start"), (5, "end")]


@pytest.mark.parametrize("new,cached,words,window,sinks", [
    ([1], [0], 1, 0, 0), ([17, 0, 33, 2], [5, 0, 100, 31], 2, 0, 0), ([70, 300], [3, 40], 10, 4, 0), ([64, 40], [0, 9], 2, 3, 12),
    ([1024], [7], 32, 0, 0), ([40, 5], [7, 2], 1, 0, 0)])
def test_draft_tree(emu, tmp_path, new, cached, words, window, sinks):
    import random
    rng = random.Random(sum(new))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    parents = np.array([x for n in new for x in tree_oracle.random_parents(rng, n, 0.7, 0.05)] + [3] * 5, np.int32)  # 5 tokens of no sequence
    T = len(parents)
    if T > 20:
        parents[[4, 11]] = [9, -5]  # no token's index, or one behind it: only cached ones are in front
    positions, seen = tree_oracle.draft_tree(parents, cu, cached, words, window, sinks)
    for order, side in ORDERS:
        raw = np.frombuffer(_run(emu, tmp_path, 0, [len(new), T, words, window, sinks], [cu, np.array(cached, np.int32), parents], order, side), np.int32)
        assert np.array_equal(raw[:T], positions)
        assert np.array_equal(raw[T:].reshape(T, words), tree_oracle.bits_of(seen, words))


@pytest.mark.parametrize("seed,batch,most,bs,more", [(1, 1, 20, 16, {}), (2, 7, 40, 8, {}), (3, 70, 30, 4, {}), (4, 5, 200, 16, dict(vocabulary=1)),
                                                    (5, 9, 130, 16, dict(holes=0.3)), (6, 6, 40, 8, dict(width=4))])
def test_accept(emu, tmp_path, seed, batch, most, bs, more):
    p = th.accept_problem(seed, batch, most, bs, **more)
    T, capacity = p["T"], 40
    free = np.arange(1000, 1000 + capacity, dtype=np.int32)
    for n_free in (3, 36, -1):
        want = tree_oracle.accept_path(p["tokens"], p["parents"], p["choices"], p["cu"], p["cached"], p["table"], bs, free, n_free)
        for gives_back in (1, 0):
            # behind the sequences two tokens of none
            arrays = [p["cu"], p["cached"], *(np.concatenate([p[k], [0, 0]]).astype(np.int32) for k in ("tokens", "parents", "choices"))]
            if gives_back:
                arrays += [p["table"], free, np.array([n_free], np.int32)]
            for order, side in ORDERS:
                raw = np.frombuffer(_run(emu, tmp_path, 1, [batch, T + 2, bs.bit_length() - 1, p["table"].shape[1], capacity, gives_back], arrays, order, side), np.int32)
                path, counts, following, lens = np.split(raw[:T + 2 + 3 * batch], [T + 2, T + 2 + batch, T + 2 + 2 * batch])
                assert np.array_equal(path, np.concatenate([want[0], [-1, -1]]))
                assert np.array_equal(counts, want[1]) and np.array_equal(following, want[2]) and np.array_equal(lens, want[3])
                if gives_back:
                    assert raw[T + 2 + 3 * batch] == want[5] and np.array_equal(raw[T + 3 + 3 * batch:], want[4])


@pytest.mark.parametrize("dtype,d,bs,n_caches", [("bf16", 128, 16, 2), ("f32", 8, 4, 3), ("f16", 40, 8, 35)])
def test_keep(emu, tmp_path, dtype, d, bs, n_caches):
    p = th.accept_problem(d, 6, 40, bs, vocabulary=2, holes=0.05)
    path = tree_oracle.accept_path(p["tokens"], p["parents"], p["choices"], p["cu"], p["cached"])[0]
    if p["new"][-1] > 2:
        path[p["cu"][-2]:p["cu"][-2] + 2] = [0, 10 ** 6]  # an index that is none ends the branch
    heads = 3
    g = torch.Generator().manual_seed(d)
    caches = [torch.randn((p["n_blocks"], heads, bs, d), generator=g).to(ah.TORCH[dtype]) for _ in range(n_caches)]
    want = tree_oracle.keep_path([c.float().numpy() for c in caches], p["table"], p["cu"], p["cached"], path)
    for order, side in ORDERS:
        raw = _run(emu, tmp_path, 2, [6, p["T"], heads, heads, d, bs, ah.CODE[dtype], p["n_blocks"], p["table"].shape[1], n_caches],
                   [p["cu"], p["cached"], p["table"], path, *[_bits(c) for c in caches]], order, side)
        got = torch.frombuffer(bytearray(raw), dtype=ah.TORCH[dtype]).float().numpy().reshape(n_caches, *caches[0].shape)
        assert np.array_equal(got, np.stack(want))


def _attend(exe, tmp_path, p, order=0, side="end", target=0, late=0):
    params = [len(p.new), p.T, p.hq, p.hkv, p.d, p.bs, ah.CODE[p.dtype], p.k_cache.shape[0], p.table.shape[1], p.window, p.sinks, p.max_new,
              int(np.float32(p.scale).view(np.int32)), p.words]
    arrays = [p.cu, np.array(p.cached, np.int32), p.table, p.positions, p.bits, _bits(p.q), _bits(p.k_cache), _bits(p.v_cache)]
    raw = _run(exe, tmp_path, 3, params, arrays, order, side, target, late)
    n, esz = p.T * p.hq * p.d, p.q.element_size()
    out = torch.frombuffer(bytearray(raw[:n * esz]), dtype=p.q.dtype).double().numpy().reshape(p.T, p.hq, p.d)
    return out, np.frombuffer(raw[n * esz:], np.float32).reshape(p.T, p.hq)


@pytest.mark.parametrize("bits", ["tree", "any"])
@pytest.mark.parametrize("name,target", [(name, target) for name in sorted(th.CASES) for target in (2, 60)])
def test_attend(emu, tmp_path, name, target, bits):
    p = th.make(11, *th.CASES[name], bits=bits)
    ref = th.reference(p)
    out, lse = _attend(emu, tmp_path, p, target=target)
    ah.check(p, out, lse, name, ref)
    for order, side, late in ((1, "start", 1), (5, "end", 0)):
        other = _attend(emu, tmp_path, p, order, side, target, late)
        assert np.array_equal(out, other[0]) and np.array_equal(lse, other[1]), f"{name}: order {order} changes the result"


@pytest.mark.parametrize("name", ["few", "chunk_window", "chunk_group", "f32"])
def test_attend_not_finite_stays_with_the_rows_that_see_it(emu, tmp_path, name):
    """Infinities and NaN in keys and values of cached and new tokens, and blocks that are missing."""
    for where in ("k_cache", "v_cache"):
        p = th.make(7, *th.CASES[name], holes=0.1, bits="any" if where == "k_cache" else "tree")
        for seq in range(len(p.new)):
            total = p.new[seq] + p.cached[seq]
            for i, bad in enumerate([float("inf"), float("nan"), -float("inf")]):
                j = total - 1 - 2 * i - (total // 2 if i == 1 else 0)
                if 0 <= j < total and 0 <= p.table[seq, j // p.bs] < p.k_cache.shape[0]:
                    block, row = p.block_row(seq, j)
                    getattr(p, where)[block, i % p.hkv, row, (5 * i + j) % p.d] = bad
        ref = th.reference(p)
        for target in (2, 30):
            out, lse = _attend(emu, tmp_path, p, target=target)
            ah.check(p, out, lse, name, ref)
