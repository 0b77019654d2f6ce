"""The entry points for trees of drafted tokens without a GPU: exported symbols, refusals and their messages, workspace sizes."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2411_19379_amd import attention as attn
from paper_2411_19379_amd import build as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # an aligned address; nothing is launched by a refused call
SHAPE = (4, 2, 64, 16, 1)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.ATTN_LIB_PATH):
        b.build_attention()
    return attn.load_library()


def test_library_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "attn_tree.h")).read()
    names = set(re.findall(r"\b(attn_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", header, flags=re.S)))
    assert names == {"attn_draft_tree", "attn_tree_workspace_bytes", "attn_attend_tree", "attn_accept_path", "attn_keep_path"}
    for n in names:
        assert hasattr(lib, n)


def _draft(lib, **kw):
    v = dict(batch=2, T=5, words=1, parents=A, cu=A, cached=A, window=0, sinks=0, positions=A, seen=A)
    v.update(kw)
    return lib.attn_draft_tree(*v.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -1), (dict(batch=4097), -4), (dict(T=-1), -1), (dict(T=1 << 30), -4), (dict(words=0), -4), (dict(words=33), -4), (dict(words=-1), -4),
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(batch=0), -1), (dict(parents=None), -1), (dict(cu=None), -1), (dict(cached=None), -1),
    (dict(positions=None), -1), (dict(seen=None), -1)])
def test_draft_refuses(lib, kw, code):
    assert _draft(lib, **kw) == code and attn.attn_last_error()


def _attend(lib, shape=SHAPE, **kw):
    v = dict(batch=2, T=3, n_blocks=8, width=4, q=A, qs=256, kc=A, vc=A, table=A, cu=A, cached=A, positions=A, seen=A, words=1, scale=0.125,
             window=0, sinks=0, max_new=0, out=A, os=256, lse=None, ws=A, ws_bytes=1 << 40)
    v.update(kw)
    return lib.attn_attend_tree(ctypes.byref(attn.AttnShape(*shape)), *v.values(), None)


@pytest.mark.parametrize("shape,kw,code", [
    ((4, 2, 96, 16, 1), dict(qs=384, os=384), -4), ((4, 3, 64, 16, 1), {}, -1), ((4, 2, 64, 16, 3), {}, -1), ((4, 2, 64, 3, 1), {}, -4),
    (None, dict(batch=-2), -1), (None, dict(batch=5000), -4), (None, dict(T=1 << 30), -4), (None, dict(batch=0), -1), (None, dict(n_blocks=0), -1),
    (None, dict(width=0), -1), (None, dict(window=-1), -1), (None, dict(sinks=-1), -1), (None, dict(max_new=-1), -1), (None, dict(scale=0.0), -1),
    (None, dict(scale=math.nan), -1), (None, dict(q=None), -1), (None, dict(kc=None), -1), (None, dict(vc=None), -1), (None, dict(table=None), -1),
    (None, dict(cu=None), -1), (None, dict(cached=None), -1), (None, dict(positions=None), -1), (None, dict(seen=None), -1), (None, dict(out=None), -1),
    (None, dict(words=0), -4), (None, dict(words=33), -4), (None, dict(q=A + 8), -6), (None, dict(kc=A + 8), -6), (None, dict(out=A + 2), -6),
    (None, dict(os=255), -1), (None, dict(ws=None), -5), (None, dict(ws_bytes=100), -5), (None, dict(ws=A + 16), -6)])
def test_attend_refuses(lib, shape, kw, code):
    assert _attend(lib, shape or SHAPE, **kw) == code and attn.attn_last_error()


def _accept(lib, **kw):
    v = dict(batch=2, bs=16, width=4, T=5, tokens=A, parents=A, choices=A, cu=A, cached=A, path=A, counts=A, next=A, lens=A, table=A, free=A, cap=9,
             n_free=A, n_free_out=2 * A)
    v.update(kw)
    return lib.attn_accept_path(*v.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -1), (dict(batch=4097), -4), (dict(T=-1), -1), (dict(T=1 << 30), -4), (dict(batch=0), -1), (dict(bs=0), -4), (dict(bs=24), -4),
    (dict(bs=2048), -4), (dict(width=0), -1), (dict(cap=-1), -1), (dict(tokens=None), -1), (dict(parents=None), -1), (dict(choices=None), -1),
    (dict(cu=None), -1), (dict(cached=None), -1), (dict(path=None), -1), (dict(counts=None), -1), (dict(next=None), -1), (dict(lens=None), -1),
    (dict(free=None), -1), (dict(n_free=None), -1), (dict(n_free_out=None), -1), (dict(n_free_out=A), -1)])
def test_accept_refuses(lib, kw, code):
    assert _accept(lib, **kw) == code and attn.attn_last_error()


def _keep(lib, shape=SHAPE, caches=(A, 2 * A), **kw):
    v = dict(batch=2, T=5, n_blocks=8, width=4, n=len(caches), caches=(ctypes.c_void_p * max(len(caches), 1))(*caches), table=A, cu=A, cached=A, path=A)
    v.update(kw)
    return lib.attn_keep_path(ctypes.byref(attn.AttnShape(*shape)), *v.values(), None)


BYTES = 8 * 2 * 16 * 64 * 2  # of a cache of 8 blocks


@pytest.mark.parametrize("shape,kw,code", [
    ((4, 2, 60, 16, 1), {}, -4), ((4, 2, 264, 16, 1), {}, -4), ((4, 0, 64, 16, 1), {}, -1), ((4, 2, 64, 16, 4), {}, -1), (None, dict(batch=-1), -1),
    (None, dict(batch=4097), -4), (None, dict(T=-1), -1), (None, dict(n_blocks=0), -1), (None, dict(n_blocks=1 << 27), -4), (None, dict(width=0), -1),
    (None, dict(n=-1), -4), (None, dict(n=257), -4), (None, dict(caches=None, n=2), -1), (None, dict(batch=0), -1), (None, dict(table=None), -1),
    (None, dict(cu=None), -1), (None, dict(cached=None), -1), (None, dict(path=None), -1)])
def test_keep_refuses(lib, shape, kw, code):
    if "caches" in kw:
        v = dict(kw)
        v.pop("caches")
        assert lib.attn_keep_path(ctypes.byref(attn.AttnShape(*SHAPE)), 2, 5, 8, 4, 2, None, A, A, A, A, None) == code
    else:
        assert _keep(lib, shape or SHAPE, **kw) == code
    assert attn.attn_last_error()


@pytest.mark.parametrize("caches,code", [((A, None), -1), ((A, A + 8), -6), ((A, A), -1), ((A, A + BYTES - 16), -1), ((2 * A, 3 * A, 2 * A - 16), -1)])
def test_keep_refuses_caches(lib, caches, code):
    assert _keep(lib, caches=caches) == code and attn.attn_last_error()


def test_null_shapes_and_empty_batches(lib):
    n = ctypes.c_size_t(7)
    shape = ctypes.byref(attn.AttnShape(*SHAPE))
    assert lib.attn_tree_workspace_bytes(None, 1, 1, 0, ctypes.byref(n)) == -1
    assert lib.attn_tree_workspace_bytes(shape, 1, 1, 0, None) == -1
    assert lib.attn_tree_workspace_bytes(shape, 1, 1, -1, ctypes.byref(n)) == -1
    assert lib.attn_tree_workspace_bytes(shape, 0, 0, 0, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.attn_keep_path(None, 1, 1, 1, 1, 0, None, A, A, A, A, None) == -1
    assert _draft(lib, T=0) == 0 and _draft(lib, batch=0, T=0) == 0
    assert _attend(lib, T=0) == 0 and _attend(lib, batch=0, T=0) == 0
    assert _accept(lib, batch=0, T=0) == 0
    assert _keep(lib, T=0) == 0 and _keep(lib, caches=()) == 0


@pytest.mark.parametrize("batch,T", [(1, 17), (64, 64), (32, 1024), (1, 1024)])
def test_workspace_holds_the_partial_results(lib, batch, T):
    """A workspace is a few partial results (128 values, maximum and sum in fp32) per query row at most, whatever max_new says."""
    for most in (0, 1, T):
        n = ctypes.c_size_t()
        assert lib.attn_tree_workspace_bytes(ctypes.byref(attn.AttnShape(32, 8, 128, 64, 1)), batch, T, most, ctypes.byref(n)) == 0
        assert n.value <= 1 << 30 and n.value % 4 == 0


def test_entry_points_refuse_host_tensors():
    if not os.path.exists(b.ATTN_BINDING_PATH):
        b.build_attention_binding()
    ints, x, cache = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 2, 64), torch.zeros(2, 2, 16, 64)
    row = ints.view(1, 2)
    for call in (lambda: attn.draft_tree(ints[:1], ints, ints[:1], 1), lambda: attn.attend_tree(x, cache, cache, row, ints, ints[:1], ints[:1], row[:, :1]),
                 lambda: attn.accept_path(ints[:1], ints[:1], ints[:1], ints, ints[:1]), lambda: attn.keep_path([cache], row, ints, ints[:1], ints[:1])):
        with pytest.raises(ValueError, match="CUDA device"):
            call()
    for call in (lambda: attn.draft_tree(None, ints, ints[:1], 1), lambda: attn.attend_tree(x, cache, cache, row, ints, ints[:1], ints[:1], None),
                 lambda: attn.accept_path(ints[:1], [0], ints[:1], ints, ints[:1]), lambda: attn.keep_path(cache, row, ints, ints[:1], ints[:1])):
        with pytest.raises((TypeError, ValueError)):
            call()
