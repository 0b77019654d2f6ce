"""The attention library's entry points without a GPU: exported symbols, refusals and their messages, workspace sizes, the
rotary table."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2411_19379_amd import attention as attn
from paper_2411_19379_amd import build as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.ATTN_LIB_PATH):
        b.build_attention()
    return attn.load_library()


def test_library_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "attn_cache.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    names = set(re.findall(r"\b(attn_[a-z0-9_]+)\s*\(", header))
    assert names == {"attn_assign_blocks", "attn_rope_append", "attn_workspace_bytes", "attn_attend", "attn_last_error"}
    for n in names:
        assert hasattr(lib, n)


A = 1 << 20  # an aligned address; nothing is launched by a refused call


def _assign(lib, **kw):
    v = dict(batch=2, bs=16, width=4, T=5, cu=A, cached=A, shared=None, tin=A, tout=A, free=A, n_free=A, cap=9, slots=A, pos=A,
             copies=A, counts=2 * A)
    v.update(kw)
    return lib.attn_assign_blocks(*v.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -1), (dict(batch=4097), -4), (dict(T=-1), -1), (dict(T=1 << 30), -4), (dict(bs=0), -4), (dict(bs=24), -4),
    (dict(bs=2048), -4), (dict(width=0), -1), (dict(cap=-1), -1), (dict(batch=0), -1), (dict(cu=None), -1), (dict(cached=None), -1),
    (dict(tin=None), -1), (dict(tout=None), -1), (dict(free=None), -1), (dict(n_free=None), -1), (dict(slots=None), -1),
    (dict(pos=None), -1), (dict(copies=None), -1), (dict(counts=None), -1), (dict(counts=A), -1), (dict(n_free=2 * A + 4), -1)])
def test_assign_refuses(lib, kw, code):
    assert _assign(lib, **kw) == code and attn.attn_last_error()


def test_assign_of_nothing(lib):
    assert _assign(lib, batch=0, T=0) == 0


def _rope(lib, shape=(4, 2, 64, 16, 1), **kw):
    v = dict(T=3, batch=1, n_blocks=8, q=A, qs=256, k=A, ks=128, v=A, vs=128, pos=A, slots=A, rot=A, most=10, dim=64, inter=0,
             copies=None, out=2 * A, kc=A, vc=A)
    v.update(kw)
    return lib.attn_rope_append(ctypes.byref(attn.AttnShape(*shape)), *v.values(), None)


@pytest.mark.parametrize("shape,kw,code", [
    ((0, 2, 64, 16, 1), {}, -1), ((4, 3, 64, 16, 1), {}, -1), ((4, 2, 64, 16, 5), {}, -1), ((4, 2, 64, 12, 1), {}, -4),
    ((4, 2, 60, 16, 1), dict(dim=48), -4), ((4, 2, 264, 16, 1), dict(qs=1056, ks=528, vs=528), -4), ((2048, 2, 64, 16, 1), {}, -4),
    (None, dict(dim=24), -4), (None, dict(dim=80), -4), (None, dict(dim=-16), -4), (None, dict(inter=2), -1), (None, dict(q=None), -1),
    (None, dict(k=None), -1), (None, dict(v=None), -1), (None, dict(slots=None), -1), (None, dict(pos=None), -1), (None, dict(rot=None), -1),
    (None, dict(most=0), -1), (None, dict(out=None), -1), (None, dict(kc=None), -1), (None, dict(vc=None), -1), (None, dict(q=A + 8), -6),
    (None, dict(k=A + 2), -6), (None, dict(kc=A + 8), -6), (None, dict(out=A + 4), -6), (None, dict(rot=A + 4), -6), (None, dict(qs=260), -6),
    (None, dict(qs=248), -1), (None, dict(ks=120), -1), (None, dict(n_blocks=0), -1), (None, dict(n_blocks=1 << 27), -4),
    (None, dict(out=A, qs=512), -1), (None, dict(T=-3), -1), (None, dict(batch=5000), -4)])
def test_rope_refuses(lib, shape, kw, code):
    assert _rope(lib, shape or (4, 2, 64, 16, 1), **kw) == code and attn.attn_last_error()


def _attend(lib, shape=(4, 2, 64, 16, 1), **kw):
    v = dict(batch=2, T=3, n_blocks=8, width=4, q=A, qs=256, kc=A, vc=A, table=A, cu=A, cached=A, scale=0.125, window=0, sinks=0,
             max_new=0, out=A, os=256, lse=None, ws=A, ws_bytes=1 << 40)
    v.update(kw)
    return lib.attn_attend(ctypes.byref(attn.AttnShape(*shape)), *v.values(), None)


@pytest.mark.parametrize("shape,kw,code", [
    ((4, 2, 96, 16, 1), dict(qs=384, os=384), -4), ((4, 0, 64, 16, 1), {}, -1), ((4, 2, 64, 16, 3), {}, -1), ((4, 2, 64, 3, 1), {}, -4),
    (None, dict(batch=-2), -1), (None, dict(batch=5000), -4), (None, dict(T=1 << 30), -4), (None, dict(T=1 << 29), -4), (None, dict(batch=0), -1),
    (None, dict(n_blocks=0), -1), (None, dict(n_blocks=1 << 27), -4), (None, dict(width=0), -1), (None, dict(window=-1), -1),
    (None, dict(sinks=-1), -1), (None, dict(max_new=-1), -1), (None, dict(scale=0.0), -1), (None, dict(scale=-1.0), -1),
    (None, dict(scale=math.inf), -1), (None, dict(scale=math.nan), -1), (None, dict(scale=3.4e38), -1), (None, dict(q=None), -1),
    (None, dict(kc=None), -1), (None, dict(vc=None), -1), (None, dict(table=None), -1), (None, dict(cu=None), -1), (None, dict(cached=None), -1),
    (None, dict(out=None), -1), (None, dict(q=A + 8), -6), (None, dict(vc=A + 8), -6), (None, dict(out=A + 2), -6), (None, dict(os=260), -6),
    (None, dict(qs=200), -1), (None, dict(os=255), -1), (None, dict(ws=None), -5), (None, dict(ws_bytes=100), -5), (None, dict(ws=A + 16), -6)])
def test_attend_refuses(lib, shape, kw, code):
    assert _attend(lib, shape or (4, 2, 64, 16, 1), **kw) == code and attn.attn_last_error()


def test_null_shapes_and_empty_batches(lib):
    n = ctypes.c_size_t(7)
    assert lib.attn_workspace_bytes(None, 1, 1, 0, ctypes.byref(n)) == -1
    assert lib.attn_workspace_bytes(ctypes.byref(attn.AttnShape(4, 2, 64, 16, 1)), 1, 1, 0, None) == -1
    assert attn.attn_workspace_bytes(attn.AttnShape(4, 2, 64, 16, 1), 0, 0) == 0
    assert _attend(lib, batch=0, T=0) == 0 and _attend(lib, T=0) == 0
    with pytest.raises(attn.AttnError) as e:
        attn.attn_workspace_bytes(attn.AttnShape(4, 2, 96, 16, 1), 1, 1)
    assert e.value.status == "ATTN_ERR_UNSUPPORTED_SHAPE" and e.value.code == -4


def test_tensors_are_checked():
    x = torch.zeros((1, 4, 64))
    with pytest.raises(ValueError):
        attn.attend(x, x, x, x, x, x)


def test_rotary_table():
    t = attn.rotary_table(100, 32, device="cpu")
    assert t.shape == (100, 2, 16) and t.dtype == torch.float32
    for p, i in ((0, 0), (1, 0), (99, 3), (57, 15)):
        angle = p * 10000.0 ** (-2.0 * i / 32)
        assert abs(float(t[p, 0, i]) - math.cos(angle)) < 1e-7 and abs(float(t[p, 1, i]) - math.sin(angle)) < 1e-7
    half = attn.rotary_table(100, 32, linear=2.0, device="cpu")
    assert torch.equal(half[2 * torch.arange(50)], t[:50])
    parts = attn.rotary_table(64, 32, by_parts=4.0, trained_positions=64, slow_turns=1.0, fast_turns=8.0, device="cpu")
    size = 0.1 * math.log(4.0) + 1.0
    # 64 positions: pair 0 turns 10 times and keeps its frequency, pair 15 a fraction of once and is divided by 4
    assert torch.allclose(parts[:, 0, 0], t[:64, 0, 0] * size, atol=1e-6)
    slow = torch.arange(64, dtype=torch.float64) * 10000.0 ** (-30 / 32) / 4
    assert torch.allclose(parts[:, 1, 15].double(), torch.sin(slow) * size, atol=1e-6)
    for kw in (dict(max_positions=0, rotary_dim=32), dict(max_positions=4, rotary_dim=24), dict(max_positions=4, rotary_dim=32, linear=0.5),
               dict(max_positions=4, rotary_dim=32, slow_turns=9.0, fast_turns=9.0)):
        with pytest.raises(ValueError):
            attn.rotary_table(device="cpu", **kw)


def test_entry_points_refuse_host_tensors():
    """There is no path without a GPU: tensors elsewhere are refused by name, and things that are no tensors by type."""
    if not os.path.exists(b.ATTN_BINDING_PATH):
        b.build_attention_binding()
    ints = torch.zeros(2, dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError)):
        attn.assign_blocks(16, 1, ints, ints[:1], ints.view(1, 2), ints, ints[:1])
    x, cache = torch.zeros(1, 2, 64), torch.zeros(2, 2, 16, 64)
    with pytest.raises((ValueError, RuntimeError)):
        attn.rope_append(x, x, x, ints[:1], ints[:1].long(), None, cache, cache)
    with pytest.raises((ValueError, RuntimeError)):
        attn.attend(x, cache, cache, ints.view(1, 2), ints, ints[:1])
    with pytest.raises(TypeError):
        attn.attend(x, cache, cache, None, ints, ints[:1])
