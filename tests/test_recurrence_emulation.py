"""The kernels of the gated recurrence on the SIMT emulator: against the definition in 64 bits, with every buffer flush against
inaccessible pages and the waves in several orders, which must not change a bit."""
from __future__ import annotations

import os
import subprocess

import numpy as np
import pytest
import torch

import rec_helpers as rh
import rec_oracle
import tree_oracle
from test_attention_emulation import _bits, _run
from test_kernel_emulation import CLANG, CSRC, EMU, ROOT, _convert

HERE = os.path.join(ROOT, "tests", "rec_emu")


def _build(d, few):
    """The emulated kernels, two channels per lane where more than `few` workgroups are left."""
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ with bf16 vector support found")
    srcs = [os.path.join(EMU, "emu_rt.cpp"), os.path.join(HERE, "emu_rec_main.cpp")]
    for name in ("rec_scan", "rec_step"):
        _convert(os.path.join(CSRC, name + ".hip"), os.path.join(d, name + ".cpp"))
        srcs.append(os.path.join(d, name + ".cpp"))
    common = open(os.path.join(CSRC, "rec_common.h")).read()
    pinned = 'asm volatile("" : "+v"(v));'  # a hint for the compiler: nothing to emulate
    assert common.count(pinned) == 1
    open(os.path.join(d, "common.h"), "w").write(common.replace(pinned, ""))
    _convert(os.path.join(d, "common.h"), os.path.join(d, "rec_common.h"))
    flags = [f"-DREC_FEW_WORKGROUPS={few}", "-std=c++17", "-O2", "-fno-strict-aliasing", "-ffp-contract=off", "-Wno-psabi", "-Wno-unused-value", "-D__popcll=__builtin_popcountll",
             "-I", d, "-I", HERE, "-I", EMU, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    procs = [subprocess.Popen([CLANG, *flags, "-c", s, "-o", os.path.join(d, f"{i}.o")], stderr=subprocess.PIPE, text=True)
             for i, s in enumerate(srcs)]
    for p in procs:
        _, err = p.communicate()
        assert p.returncode == 0, err[-3000:]
    exe = os.path.join(d, "emu_rec_main")
    subprocess.run([CLANG, *[os.path.join(d, f"{i}.o") for i in range(len(srcs))], "-o", exe], check=True)
    return exe


@pytest.fixture(scope="session")
def emu(tmp_path_factory):
    return _build(str(tmp_path_factory.mktemp("rec_emu")), 0)


@pytest.fixture(scope="session")
def emu_few(tmp_path_factory):
    return _build(str(tmp_path_factory.mktemp("rec_emu_few")), 1 << 20)


ORDERS = [(1, "start"), (5, "end")]


def _rows(t, gap):
    """Rows with `gap` elements between them, the last one's end the end of all."""
    if not t.numel():
        return b""
    wide = torch.full((t.shape[0], t.shape[1] + gap), float("nan"), dtype=t.dtype)
    wide[:, :t.shape[1]] = t
    return _bits(wide.reshape(-1)[:wide.numel() - gap])


def _common(p, gap):
    params = [p.C, rh.CODE[p.dtype], int(np.float32(p.sharpness).view(np.int32)), len(p.lens), p.T, gap]
    return params, [p.cu, _rows(p.x, gap), _rows(p.r, gap), _rows(p.i, gap), p.decay.numpy()]


def _take(raw, sizes, dtype):
    """The parts of the output: True: of the type, False: fp32."""
    esz, out, at = 4 if dtype == "f32" else 2, [], 0
    for of_type, shape in sizes:
        n = int(np.prod(shape))
        kind, size = (rh.TORCH[dtype], esz) if of_type else (torch.float32, 4)
        out.append(torch.frombuffer(bytearray(raw[at:at + n * size]) or bytearray(size), dtype=kind)[:n].double().numpy().reshape(shape))
        at += n * size
    assert at == len(raw)
    return out


def _untouched(a):
    """Whether an array of the output was not written."""
    return a.size == 0 or np.isnan(a).all() or np.all(a == a.flat[0]) and abs(a.flat[0]) > 1e4  # (the pattern is a NaN of fp16)


def _scan(exe, tmp_path, p, ckpt=(), save=True, gap=0, order=0, side="end"):
    params, arrays = _common(p, gap)
    if p.init is not None:
        arrays.append(p.init.numpy())
    arrays.append(np.array(ckpt, np.int32))
    raw = _run(exe, tmp_path, 0, params + [int(p.init is not None), len(ckpt), int(save)], arrays, order, side)
    batch = len(p.lens)
    sizes = [(True, (p.T, p.C)), (False, (batch, p.C)), (False, (len(ckpt), p.C))] + [(False, (-(-p.T // 8), p.C))] * save
    return _take(raw, sizes, p.dtype)


@pytest.mark.parametrize("name", sorted(rh.CASES))
def test_scan(emu, tmp_path, name):
    C, dtype, lens, more = rh.CASES[name]
    p = rh.make(5, C, dtype, lens, **more)
    ckpt = [0, p.T - 1, p.T // 2, p.T // 3, p.T // 2, -1, p.T + 5, 2 ** 31 - 1]
    y, final, states, saved = _scan(emu, tmp_path, p, ckpt)
    rh.check_scan(p, y, final, ckpt, states)
    assert _untouched(y[:p.cu[0]]) and _untouched(y[p.cu[-1]:])
    for order, side in ORDERS:
        other = _scan(emu, tmp_path, p, ckpt, order=order, side=side)
        # what is saved for tokens of no sequence says nothing
        assert all(np.array_equal(a, b) for a, b in zip((y, final, states), other)), order


def test_scan_rows_of_a_projection(emu, tmp_path):
    """Odd distances between rows: a channel per lane, the same values."""
    p = rh.make(2, 64, "bf16", [70, 30])
    want = _scan(emu, tmp_path, p)
    for gap in (3, 8):
        got = _scan(emu, tmp_path, p, gap=gap)
        assert all(np.array_equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("where", ["x", "r", "i", "init"])
def test_scan_not_finite_stays_in_its_sequence(emu, tmp_path, where):
    for dtype in ("f32", "bf16"):
        p = rh.make(3, 66, dtype, [40, 100, 90, 1, 30])
        if where == "init":
            p.init[1, 3], p.init[2, 65] = float("inf"), float("nan")
        else:
            v = getattr(p, where)
            v[45, 3], v[150, 65], v[229, 7] = float("inf") if where == "x" else float("nan"), float("nan"), float("nan")
        h, want_final = rh.reference(p)
        y, final, _, _ = _scan(emu, tmp_path, p)
        assert np.array_equal(np.isfinite(y), np.isfinite(h)) and np.array_equal(np.isfinite(final), np.isfinite(want_final))


@pytest.mark.parametrize("name", ["chunks", "groups"])
def test_one_channel_per_lane_is_two(emu, emu_few, tmp_path, name):
    C, dtype, lens, more = rh.CASES[name]
    p = rh.make(8, C, dtype, lens, **more)
    for call in (lambda exe: _scan(exe, tmp_path, p, [0, p.T // 2]), lambda exe: _grads(exe, tmp_path, p)):
        for a, b in zip(call(emu), call(emu_few)):
            assert np.array_equal(a, b, equal_nan=True)


def _grads(exe, tmp_path, p, dy=True, d_final=True, init=True, gap=0, order=0, side="end"):
    params, arrays = _common(p, gap)
    if p.init is not None:
        arrays.append(p.init.numpy())
    arrays += [_bits(p.dy)] * dy + [p.d_final.numpy()] * d_final
    raw = _run(exe, tmp_path, 1, params + [int(p.init is not None), int(dy), int(d_final), int(init)], arrays, order, side)
    return _take(raw, [(True, (p.T, p.C))] * 3 + [(False, (p.C,))] + [(False, (len(p.lens), p.C))] * init, p.dtype) + [None] * (not init)


@pytest.mark.parametrize("name", sorted(rh.CASES))
def test_grads(emu, tmp_path, name):
    C, dtype, lens, more = rh.CASES[name]
    p = rh.make(6, C, dtype, lens, **more)
    got = _grads(emu, tmp_path, p)
    rh.check_grads(p, got)
    for order, side in ORDERS:
        other = _grads(emu, tmp_path, p, order=order, side=side)
        assert all(np.array_equal(a, b) for a, b in zip(got, other)), order


@pytest.mark.parametrize("dy,d_final,init", [(False, True, True), (True, False, False), (False, False, True)])
def test_grads_of_some_outputs(emu, tmp_path, dy, d_final, init):
    p = rh.make(8, 64, "bf16", [70, 0, 20])
    rh.check_grads(p, _grads(emu, tmp_path, p, dy, d_final, init), dy, d_final, init)


def test_grads_at_gates_that_are_shut(emu, tmp_path):
    """sigmoid(r) down to 0: 1 - a^2 vanishes, and the gradients through it go to their limit 0."""
    p = rh.make(9, 64, "f32", [40])
    p.r[:] = torch.linspace(-120.0, 30.0, 40)[:, None]
    p.i[:] = torch.linspace(-100.0, 100.0, 64)
    y, final, _, _ = _scan(emu, tmp_path, p)
    got = _grads(emu, tmp_path, p)
    for a in (y, final, *got):
        assert np.isfinite(a).all()
    rh.check_scan(p, y, final)
    shut = p.r[:, 0].numpy() < -90
    assert np.all(got[1][shut] == 0)
    open_ = np.abs(p.r[:, 0].numpy()) < 20
    want = rec_oracle.grads(*rh.arrays(p), p.cu, p.sharpness, p.init.double().numpy(), p.dy.double().numpy(), p.d_final.double().numpy())
    assert np.allclose(got[0][open_], want[0][open_], rtol=1e-4, atol=1e-6) and np.allclose(got[1][open_], want[1][open_], rtol=1e-3, atol=1e-5)


@pytest.mark.parametrize("C,dtype,batch,gap", [(64, "bf16", 3, 0), (1, "f32", 5, 0), (301, "f16", 2, 3), (258, "f32", 1, 2)])
def test_step(emu, tmp_path, C, dtype, batch, gap):
    p = rh.make(4, C, dtype, [1] * batch)
    for order, side in [(0, "end")] + ORDERS:
        params, arrays = _common(p, gap)
        raw = _run(emu, tmp_path, 2, params, arrays + [p.init.numpy()], order, side)
        y, states = _take(raw, [(True, (batch, C)), (False, (batch, C))], dtype)
        rh.check_scan(p, y, states)


@pytest.mark.parametrize("C,dtype,lens,lead,behind", [(64, "bf16", [1, 0, 17], 0, 0), (70, "f32", [90, 150, 3], 0, 9), (65, "f16", [8, 9], 4, 0), (2, "bf16", [200], 0, 0)])
def test_step_tree(emu, tmp_path, C, dtype, lens, lead, behind):
    import random
    p = rh.make(4, C, dtype, lens, lead=lead, behind=behind)
    rng = random.Random(C)
    parents = np.array([-1] * lead + [x for n in lens for x in tree_oracle.random_parents(rng, n, 0.6, 0.1)] + [0] * behind, np.int32)
    path = np.full(p.T, -1, np.int32)
    counts = np.zeros(len(lens), np.int32)
    for b, n in enumerate(lens):
        line = tree_oracle.branch(parents[p.cu[b]:p.cu[b + 1]].tolist(), n - 1)[::-1] if n else []
        path[p.cu[b]:p.cu[b] + len(line)], counts[b] = line, len(line)
    h = rec_oracle.tree(*rh.arrays(p), p.init.double().numpy(), p.cu, parents, p.sharpness)
    e = rh.Errors(p)
    size, off = np.zeros(h.shape), np.zeros(h.shape)
    for b in range(len(lens)):
        for k in range(lens[b]):
            t, q = p.cu[b] + k, parents[p.cu[b] + k]
            s, o = (size[p.cu[b] + q], off[p.cu[b] + q]) if q >= 0 else (np.abs(p.init[b].double().numpy()), 0.0)
            size[t], off[t] = e.a[t] * s + e.added[t], e.a[t] * (o + (e.a_off[t] + 4) * s) + e.added_off[t] * e.added[t]
    bound = off * rh.UNIT + 1e-30
    for order, side in [(0, "end")] + ORDERS:
        params, arrays = _common(p, 0)
        raw = _run(emu, tmp_path, 3, params, arrays + [p.init.numpy(), parents, path, counts], order, side)
        y, nodes, states = _take(raw, [(True, (p.T, C)), (False, (p.T, C)), (False, (len(lens), C))], dtype)
        inside = slice(int(p.cu[0]), int(p.cu[-1]))
        rh.check("nodes", nodes[inside], h[inside], bound[inside])
        tiny = 2.0 ** -25 if dtype == "f16" else 1e-38
        rh.check("y", y[inside], h[inside], (bound + rh.HALF_ULP[dtype] * (np.abs(h) + bound) + tiny)[inside])
        assert _untouched(y[:p.cu[0]]) and _untouched(nodes[p.cu[-1]:])
        for b, n in enumerate(lens):
            assert np.array_equal(states[b], nodes[p.cu[b] + n - 1] if n else p.init[b].double().numpy())
