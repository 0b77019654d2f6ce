"""The gated recurrence's entry points without a GPU: exported symbols, refusals and their messages, workspace sizes."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2411_19379_amd import build as b
from paper_2411_19379_amd import recurrence as rec

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # an aligned address; nothing is launched by a refused call
SHAPE = (64, 1, 8.0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.REC_LIB_PATH):
        b.build_recurrence()
    return rec.load_library()


def test_library_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "gated_recurrence.h")).read()
    names = set(re.findall(r"\b(rec_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", header, flags=re.S)))
    assert names == {"rec_workspace_bytes", "rec_scan", "rec_scan_grads", "rec_step", "rec_step_tree", "rec_keep_states", "rec_last_error"}
    for n in names:
        assert hasattr(lib, n)
    assert f"#define REC_SAVED_EVERY {rec.REC_SAVED_EVERY}\n" in header


INPUTS = dict(x=A, xs=64, r=A, rs=64, i=A, is_=64, decay=A)


def _call(f, shape, v, kw):
    unknown = set(kw) - set(v)
    assert not unknown, unknown
    v = dict(v, **kw)
    return f(ctypes.byref(rec.RecShape(*shape)), *v.values(), None)


def _scan(lib, shape=SHAPE, **kw):
    return _call(lib.rec_scan, shape, dict(batch=2, T=100, **INPUTS, cu=A, init=A, ckpt=A, n_ckpt=3, y=A, ys=64, final=A, ckpt_states=A, saved=A, ws=A,
                                           ws_bytes=1 << 40), kw)


def _grads(lib, shape=SHAPE, **kw):
    return _call(lib.rec_scan_grads, shape, dict(batch=2, T=100, **INPUTS, cu=A, init=A, saved=A, dy=A, dys=64, d_final=A, dx=A, dr=A, di=A, d_decay=A,
                                                 d_init=A, ws=A, ws_bytes=1 << 40), kw)


def _step(lib, shape=SHAPE, **kw):
    return _call(lib.rec_step, shape, dict(batch=2, **INPUTS, states=A, y=A, ys=64), kw)


def _tree(lib, shape=SHAPE, **kw):
    return _call(lib.rec_step_tree, shape, dict(batch=2, T=100, **INPUTS, states=A, cu=A, parents=A, y=A, ys=64, nodes=A), kw)


SHAPES = [((0, 1, 8.0), -1), ((-3, 1, 8.0), -1), ((1 << 21, 1, 8.0), -4), ((64, 3, 8.0), -1), ((64, -1, 8.0), -1), ((64, 1, 0.0), -1), ((64, 1, -8.0), -1),
          ((64, 1, math.inf), -1), ((64, 1, math.nan), -1)]


@pytest.mark.parametrize("shape,code", SHAPES)
def test_shapes_are_checked(lib, shape, code):
    for call in (_scan, _grads, _step, _tree):
        assert call(lib, shape) == code and rec.rec_last_error()
    assert lib.rec_workspace_bytes(ctypes.byref(rec.RecShape(*shape)), 1, 1, 0, ctypes.byref(ctypes.c_size_t())) == code


BATCHES = [(dict(batch=-1), -1), (dict(batch=4097), -4)]
TOKENS = [(dict(T=-1), -1), (dict(T=1 << 30), -4), (dict(batch=0), -1)]
ROWS = [(dict(x=None), -1), (dict(r=None), -1), (dict(i=None), -1), (dict(decay=None), -1), (dict(xs=63), -1), (dict(rs=0), -1), (dict(is_=-64), -1),
        (dict(xs=(1 << 22) + 2), -1), (dict(x=A + 1), -6), (dict(r=A + 1), -6), (dict(i=A + 1), -6), (dict(decay=A + 2), -6)]


@pytest.mark.parametrize("kw,code", BATCHES + TOKENS + ROWS + [
    (dict(cu=None), -1), (dict(n_ckpt=-1), -1), (dict(ckpt=None), -1), (dict(ckpt_states=None), -1), (dict(ys=63), -1), (dict(y=A + 1), -6),
    (dict(init=A + 2), -6), (dict(final=A + 2), -6), (dict(ckpt_states=A + 2), -6), (dict(saved=A + 2), -6), (dict(ws=A + 16), -6), (dict(batch=0, T=0), -1)])
def test_scan_refuses(lib, kw, code):
    assert _scan(lib, **kw) == code and rec.rec_last_error()


def test_scan_refuses_small_workspaces(lib):
    need = rec.rec_workspace_bytes(rec.RecShape(4096, 1, 8.0), 2, 30000)
    assert need > 0
    big = dict(T=30000, xs=4096, rs=4096, is_=4096, ys=4096)
    assert _scan(lib, (4096, 1, 8.0), ws_bytes=need - 1, **big) == -5 and _scan(lib, (4096, 1, 8.0), ws=None, **big) == -5


@pytest.mark.parametrize("kw,code", BATCHES + TOKENS + ROWS + [
    (dict(cu=None), -1), (dict(dx=None), -1), (dict(dr=None), -1), (dict(di=None), -1), (dict(d_decay=None), -1), (dict(dys=63), -1), (dict(dy=A + 1), -6),
    (dict(dx=A + 1), -6), (dict(init=A + 2), -6), (dict(saved=A + 2), -6), (dict(d_final=A + 2), -6), (dict(d_decay=A + 2), -6), (dict(d_init=A + 2), -6),
    (dict(ws=None), -5), (dict(ws_bytes=8), -5), (dict(ws=A + 16), -6)])
def test_grads_refuse(lib, kw, code):
    assert _grads(lib, **kw) == code and rec.rec_last_error()


@pytest.mark.parametrize("kw,code", BATCHES + ROWS + [(dict(states=None), -1), (dict(y=None), -1), (dict(ys=63), -1), (dict(y=A + 1), -6),
                                                      (dict(states=A + 2), -6)])
def test_step_refuses(lib, kw, code):
    assert _step(lib, **kw) == code and rec.rec_last_error()


@pytest.mark.parametrize("kw,code", BATCHES + TOKENS + ROWS + [(dict(states=None), -1), (dict(cu=None), -1), (dict(parents=None), -1), (dict(y=None), -1),
                                                               (dict(nodes=None), -1), (dict(ys=63), -1), (dict(states=A + 2), -6), (dict(nodes=A + 2), -6)])
def test_tree_refuses(lib, kw, code):
    assert _tree(lib, **kw) == code and rec.rec_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(channels=0), -4), (dict(channels=1 << 21), -4), (dict(batch=-1), -1), (dict(batch=4097), -4), (dict(T=-1), -1), (dict(T=1 << 30), -4),
    (dict(batch=0), -1), (dict(states=None), -1), (dict(nodes=None), -1), (dict(cu=None), -1), (dict(path=None), -1), (dict(counts=None), -1),
    (dict(states=A + 2), -6), (dict(nodes=A + 1), -6)])
def test_keep_refuses(lib, kw, code):
    v = dict(channels=64, batch=2, T=5, states=A, nodes=A, cu=A, path=A, counts=A)
    assert lib.rec_keep_states(*dict(v, **kw).values(), None) == code and rec.rec_last_error()


def test_workspaces(lib):
    n = ctypes.c_size_t(7)
    shape = ctypes.byref(rec.RecShape(*SHAPE))
    assert lib.rec_workspace_bytes(None, 1, 1, 0, ctypes.byref(n)) == -1 and lib.rec_workspace_bytes(shape, 1, 1, 0, None) == -1
    assert lib.rec_workspace_bytes(shape, 1, 1, 3, ctypes.byref(n)) == -1 and lib.rec_workspace_bytes(shape, 1, 1, -1, ctypes.byref(n)) == -1
    # tokens times channels whose workgroups would not be counted in 31 bits
    assert lib.rec_workspace_bytes(ctypes.byref(rec.RecShape(1 << 20, 1, 8.0)), 1, (1 << 30) - 1, 0, ctypes.byref(n)) == -4
    for grads in (0, 1, 2):
        last = 0
        for T in (0, 1, 17, 1000, 40000):
            need = rec.rec_workspace_bytes(rec.RecShape(2560, 1, 8.0), 4, T, grads)
            assert need >= last and need % 4 == 0
            last = need
    # `saved` computed by the call itself: its rows are in the workspace
    T, C = 4096, 256
    more = rec.rec_workspace_bytes(rec.RecShape(C, 1, 8.0), 1, T, 2) - rec.rec_workspace_bytes(rec.RecShape(C, 1, 8.0), 1, T, 1)
    assert more >= T // rec.REC_SAVED_EVERY * C * 4
    with pytest.raises(rec.RecError) as e:
        rec.rec_workspace_bytes(rec.RecShape(1 << 21, 1, 8.0), 1, 1)
    assert e.value.status == "REC_ERR_UNSUPPORTED_SHAPE" and e.value.code == -4


def test_empty_batches(lib):
    assert _scan(lib, batch=0, T=0, n_ckpt=0) == 0 and _step(lib, batch=0) == 0 and _tree(lib, T=0) == 0 and _tree(lib, batch=0, T=0) == 0
    assert lib.rec_keep_states(64, 0, 0, A, A, A, A, A, None) == 0


def test_entry_points_refuse_host_tensors():
    if not os.path.exists(b.REC_BINDING_PATH):
        b.build_recurrence_binding()
    x, decay, states, ints = torch.zeros(3, 8), torch.zeros(8), torch.zeros(2, 8), torch.zeros(3, dtype=torch.int32)
    for grad in (False, True):
        leaf = x.clone().requires_grad_(grad)
        with pytest.raises(ValueError, match="CUDA device"):
            rec.gated_scan(leaf, x, x, decay, ints)
    with pytest.raises(ValueError, match="not differentiable"):
        rec.gated_scan(leaf, x, x, decay, ints, ckpt=ints)
    with pytest.raises(ValueError, match="not differentiable"):
        rec.gated_scan(x, x, x, decay, ints, init_states=states.clone().requires_grad_(), out=x)
    with pytest.raises(ValueError, match="out requires grad"):
        rec.gated_scan(x, x, x, decay, ints, out=leaf)
    for call in (lambda: rec.gated_scan_grads(x, None, x, x, x, decay, ints), lambda: rec.gated_step(x[:2], x[:2], x[:2], decay, states),
                 lambda: rec.gated_step_tree(x, x, x, decay, states, ints, ints), lambda: rec.keep_states(states, x, ints, ints, ints[:2])):
        with pytest.raises(ValueError, match="CUDA device"):
            call()
    with pytest.raises(ValueError, match="x requires grad"):
        rec.gated_step(leaf[:2], x[:2], x[:2], decay, states)
    with pytest.raises(ValueError, match="states requires grad"):
        rec.gated_step_tree(x, x, x, decay, states.clone().requires_grad_(), ints, ints)
    with pytest.raises(TypeError):
        rec.gated_step(x, x, None, decay, states)
