"""Sizes beyond what a launch of the gated recurrence can number, without a GPU: refused in front of the first launch."""
import ctypes

import pytest

from paper_2411_19379_amd import recurrence as rec
from test_recurrence_host import A, _grads, _scan, lib  # noqa: F401 (a fixture)

# A launch numbers its threads in 32 bits, and a workgroup has 512: at most 2^23 - 1 workgroups, of 64 channels (128 where rows are
# aligned to pairs) and 128 tokens, 64 in the backward pass.
MOST = (1 << 23) - 1


# `fits`: the call goes on to its workspace, which is missing
@pytest.mark.parametrize("call,C,dtype,T,fits", [
    (_scan, 64, 1, MOST * 128, True), (_scan, 64, 1, MOST * 128 + 1, False), (_scan, 1, 0, (1 << 30) - 1, False),
    (_scan, 128, 1, MOST * 128, True), (_scan, 129, 1, MOST * 64, False), (_scan, 130, 1, MOST // 2 * 128, True), (_scan, 130, 1, MOST // 2 * 128 + 1, False),
    (_grads, 64, 1, MOST * 64, True), (_grads, 64, 1, MOST * 64 + 1, False), (_grads, 1, 2, 1 << 29, False), (_grads, 1, 2, (1 << 30) - 1, False),
    (_grads, 128, 1, MOST * 64, True), (_grads, 128, 0, MOST * 64, False), (_grads, 128, 0, MOST // 2 * 64, True)])
def test_more_workgroups_than_a_launch_has(lib, call, C, dtype, T, fits):  # noqa: F811
    wide = dict(xs=C, rs=C, is_=C, **({"ys": C} if call is _scan else {"dys": C}))
    for saved in (A, None):
        assert call(lib, (C, dtype, 8.0), T=T, ws=None, saved=saved, **wide) == (-5 if fits else -4)
        assert ("workspace" if fits else "workgroups") in rec.rec_last_error()
    n = ctypes.c_size_t()
    for grads in (0,) if call is _scan else (1, 2):
        assert lib.rec_workspace_bytes(ctypes.byref(rec.RecShape(C, dtype, 8.0)), 2, T, grads, ctypes.byref(n)) == (0 if fits else -4)


def test_rows_that_are_not_aligned_to_pairs_need_more_workgroups(lib):  # noqa: F811
    shape, T = (128, 1, 8.0), MOST // 2 * 128 + 1
    rows = dict(xs=128, rs=128, is_=128)
    assert _scan(lib, shape, T=T, ws=None, ys=128, **rows) == -5
    for more in (dict(xs=129), dict(x=A + 2), dict(y=A + 2), dict(init=A + 4)):
        assert _scan(lib, shape, T=T, ws=None, **{**rows, "ys": 128, **more}) == -4
    T = MOST // 2 * 64 + 1
    assert _grads(lib, shape, T=T, ws=None, dys=128, **rows) == -5
    for more in (dict(xs=129), dict(dy=A + 2), dict(dx=A + 2), dict(d_init=A + 4)):
        assert _grads(lib, shape, T=T, ws=None, **{**rows, "dys": 128, **more}) == -4
