"""Binding of the attention layers' operators (`include/attn_cache.h`, `include/attn_tree.h`): argument marshalling only.

    step = assign_blocks(block_size, total_tokens, cu_seqlens, cached_lens, table, free_blocks, n_free)   # once per step
    q = rope_append(q, k, v, step.positions, step.slots, rotary, k_cache, v_cache, copies=step.copies)    # once per layer
    out = attend(q, k_cache, v_cache, step.table, cu_seqlens, cached_lens)

A step that checks trees of drafted tokens has, with `step` as above,

    tree = draft_tree(parents, cu_seqlens, cached_lens, max_new)                                          # once per step
    q = rope_append(q, k, v, tree.positions, step.slots, rotary, k_cache, v_cache, copies=step.copies)    # once per layer
    out = attend_tree(q, k_cache, v_cache, step.table, cu_seqlens, cached_lens, tree.positions, tree.seen, max_new=max_new)
    kept = accept_path(tokens, parents, choices, cu_seqlens, cached_lens, ...)                            # behind the model
    keep_path(caches, step.table, cu_seqlens, cached_lens, kept.path)                                     # all layers

All of it is enqueued on the current torch stream, nothing waits for the GPU, and lengths are read there; outputs and the
workspace are torch tensors.  There is no CPU fallback: loading raises if the library has not been built.  There is no backward
pass either: where a graph is recorded, tensors that require grad are refused (serve under `torch.no_grad()`), and tensors with a
tangent of forward-mode differentiation always.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple, Optional

import torch  # owns device memory and streams; its HIP runtime is the one the library has to bind to

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libattn_cache.so")
_lib = None

ATTN_DT_F32, ATTN_DT_BF16, ATTN_DT_F16 = 0, 1, 2

_STATUS = {0: "ATTN_OK", -1: "ATTN_ERR_INVALID_ARG", -4: "ATTN_ERR_UNSUPPORTED_SHAPE",
           -5: "ATTN_ERR_WORKSPACE_TOO_SMALL", -6: "ATTN_ERR_MISALIGNED", -7: "ATTN_ERR_HIP"}


class AttnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_STATUS.get(code, code)}: {msg}")
        self.code = code
        self.status = _STATUS.get(code, str(code))


class AttnShape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("io_dtype", ctypes.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libattn_cache.so (built by `python -m paper_2411_19379_amd.build`); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} is not built: run `python -m paper_2411_19379_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    shape = ctypes.POINTER(AttnShape)
    lib.attn_assign_blocks.restype = ctypes.c_int
    lib.attn_assign_blocks.argtypes = [i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.attn_rope_append.restype = ctypes.c_int
    lib.attn_rope_append.argtypes = [shape, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp, vp, vp, i32, i32, i32, vp, vp, vp,
                                     vp, vp]
    lib.attn_workspace_bytes.restype = ctypes.c_int
    lib.attn_workspace_bytes.argtypes = [shape, i32, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.attn_attend.restype = ctypes.c_int
    lib.attn_attend.argtypes = [shape, i32, i64, i32, i32, vp, i64, vp, vp, vp, vp, vp, ctypes.c_float, i32, i32, i32, vp,
                                i64, vp, vp, ctypes.c_size_t, vp]
    lib.attn_tree_workspace_bytes.restype = ctypes.c_int
    lib.attn_tree_workspace_bytes.argtypes = [shape, i32, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.attn_draft_tree.restype = ctypes.c_int
    lib.attn_draft_tree.argtypes = [i32, i64, i32, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.attn_attend_tree.restype = ctypes.c_int
    lib.attn_attend_tree.argtypes = [shape, i32, i64, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp, vp, i32, ctypes.c_float, i32, i32,
                                     i32, vp, i64, vp, vp, ctypes.c_size_t, vp]
    lib.attn_accept_path.restype = ctypes.c_int
    lib.attn_accept_path.argtypes = [i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.attn_keep_path.restype = ctypes.c_int
    lib.attn_keep_path.argtypes = [shape, i32, i64, i32, i32, i32, ctypes.POINTER(vp), vp, vp, vp, vp, vp]
    lib.attn_last_error.restype = ctypes.c_char_p
    lib.attn_last_error.argtypes = []
    _lib = lib
    return lib


def attn_last_error() -> str:
    return load_library().attn_last_error().decode()


def _check(rc: int):
    if rc != 0:
        raise AttnError(rc, attn_last_error())


def attn_workspace_bytes(shape: AttnShape, batch: int, total_tokens: int, max_new: int = 0) -> int:
    n = ctypes.c_size_t()
    _check(load_library().attn_workspace_bytes(ctypes.byref(shape), batch, total_tokens, max_new, ctypes.byref(n)))
    return n.value


_binding = None


def _native():
    """The compiled binding (csrc/attn_binding.cpp), which checks tensors and allocates outputs; raises if it is not built."""
    global _binding
    if _binding is None:
        load_library()
        try:
            from . import _attn_binding
        except ImportError as e:
            raise ImportError(f"the attention binding is not built or does not fit this torch ({e}): "
                              "run `python -m paper_2411_19379_amd.build`") from e
        _attn_binding.set_error_class(AttnError)
        _binding = _attn_binding
    return _binding


class Step(NamedTuple):
    """What `assign_blocks` returns; device tensors."""
    table: "torch.Tensor"      # [batch, max_blocks] int32
    slots: "torch.Tensor"      # [total_tokens] int64, -1: no block
    positions: "torch.Tensor"  # [total_tokens] int32
    copies: "torch.Tensor"     # [batch, 4] int32: from block, to block, rows, 0
    counts: "torch.Tensor"     # [2] int32: free blocks left, blocks missing in this call (list empty, or row too short)


def assign_blocks(block_size: int, total_tokens: int, cu_seqlens, cached_lens, table, free_blocks, n_free,
                  shared_tail=None, in_place: bool = False) -> Step:
    """Blocks, slots and positions of the new tokens of a batch.  `n_free` is a device int32 tensor of one value; the
    next step's is `counts[:1]` of this one.  `in_place` extends the rows of `table`, else they are written to a new one."""
    return Step._make((_binding or _native()).assign_blocks(block_size, total_tokens, cu_seqlens, cached_lens, table, free_blocks,
                                                            n_free, shared_tail, in_place))


def rotary_table(max_positions: int, rotary_dim: int, base: float = 10000.0, *, linear: float = 1.0,
                 by_parts: float = 1.0, trained_positions: int = 4096, slow_turns: float = 1.0, fast_turns: float = 32.0,
                 device="cuda"):
    """[max_positions, 2, rotary_dim / 2] fp32: cos and sin of position * base^(-2 i / rotary_dim), in 64 bits and rounded
    once.  For contexts longer than the `trained_positions`: `linear` divides every position by that factor; `by_parts` (the
    interpolation by parts of arXiv 2309.00071) divides by that factor the frequencies that turn fewer than `slow_turns` times over
    the trained positions, keeps those that turn more than `fast_turns` times, goes over linearly between, and scales cos and
    sin by 0.1 ln(by_parts) + 1."""
    if max_positions < 1 or rotary_dim < 16 or rotary_dim % 16:
        raise ValueError("max_positions must be positive, rotary_dim a positive multiple of 16")
    if linear < 1.0 or by_parts < 1.0 or not slow_turns < fast_turns:
        raise ValueError("factors are at least 1, slow_turns less than fast_turns")
    freq = base ** (-2.0 * torch.arange(rotary_dim // 2, dtype=torch.float64) / rotary_dim)
    keep = ((trained_positions * freq / (2.0 * math.pi) - slow_turns) / (fast_turns - slow_turns)).clamp(0.0, 1.0)
    freq = (freq * keep + freq / by_parts * (1.0 - keep)) / linear
    angle = torch.arange(max_positions, dtype=torch.float64)[:, None] * freq
    size = 0.1 * math.log(by_parts) + 1.0
    return torch.stack([angle.cos() * size, angle.sin() * size], 1).float().contiguous().to(device)


def rope_append(q, k, v, positions, slots, rotary, k_cache, v_cache, *, interleaved: bool = False, copies=None, q_out=None):
    """Rotary positions on q and k, k and v into the cache; returns the turned q [tokens, n_q_heads, head_dim].
    q, k and v may be parts of one projection's rows.  `rotary` is a `rotary_table` or None, `copies` comes from
    `assign_blocks` where sequences share their tails."""
    return (_binding or _native()).rope_append(q, k, v, positions, slots, rotary, k_cache, v_cache, interleaved, copies, q_out)


def attend(q, k_cache, v_cache, table, cu_seqlens, cached_lens, *, scale: Optional[float] = None, window: int = 0,
           sinks: int = 0, max_new: int = 0, out=None, return_lse: bool = False):
    """Attention of the new tokens over the cache.  Returns out [tokens, n_q_heads, head_dim], with `return_lse` also the
    log of the sum of exponentials [tokens, n_q_heads].  `scale` is 1 / sqrt(head_dim) if not given; `max_new`, the largest
    number of new tokens of any sequence, picks the faster kernel (0: not known)."""
    return (_binding or _native()).attend(q, k_cache, v_cache, table, cu_seqlens, cached_lens, scale, window, sinks, max_new, out,
                                          return_lse)


class Tree(NamedTuple):
    """What `draft_tree` returns; device tensors."""
    positions: "torch.Tensor"  # [total_tokens] int32
    seen: "torch.Tensor"       # [total_tokens, ceil(max_new / 32)] int32: bit j: the token sees new token j of its sequence


def draft_tree(parents, cu_seqlens, cached_lens, max_new: int, *, window: int = 0, sinks: int = 0) -> Tree:
    """Positions and visibility of a step's trees.  `parents` [tokens] int32: the index in its sequence of the token in front of
    each, -1 where only cached ones are; `max_new` at least the longest sequence's new tokens, at most 1024.  Layers with a
    sliding window take bits of their own."""
    return Tree._make((_binding or _native()).draft_tree(parents, cu_seqlens, cached_lens, max_new, window, sinks))


def attend_tree(q, k_cache, v_cache, table, cu_seqlens, cached_lens, positions, seen, *, scale: Optional[float] = None,
                window: int = 0, sinks: int = 0, max_new: int = 0, out=None, return_lse: bool = False):
    """`attend` where the new tokens are trees: cached keys are seen by `positions`, a sequence's new tokens by the bits of
    `seen`, which need not come from `draft_tree`: a row may have any bits up to its own token's, or none.  Without `max_new` all
    tokens are taken to be one sequence's, as a rule for a kernel that is made for more rows (32 trees of 16 to 64 tokens over
    114453 cached keys 229 us, with it 162)."""
    return (_binding or _native()).attend_tree(q, k_cache, v_cache, table, cu_seqlens, cached_lens, positions, seen, scale, window,
                                               sinks, max_new, out, return_lse)


class Accepted(NamedTuple):
    """What `accept_path` returns; device tensors of int32."""
    path: "torch.Tensor"         # [total_tokens]: at cu_seqlens[b] + k the k-th kept token of sequence b, -1 behind the last
    counts: "torch.Tensor"       # [batch]: kept tokens
    next_tokens: "torch.Tensor"  # [batch]: the token chosen behind the last kept one
    kept_lens: "torch.Tensor"    # [batch]: cached tokens of the next step
    n_free: Optional["torch.Tensor"]  # [1]: length of the free list with the blocks that came back; None without a table


def accept_path(tokens, parents, choices, cu_seqlens, cached_lens, *, block_size: int = 0, table=None, free_blocks=None,
                n_free=None) -> Accepted:
    """The branch of each tree that `choices` agrees with: its first token, and from there on the first child that is the token
    chosen behind its parent.  With `table`, `free_blocks` and `n_free` (as `assign_blocks` left them: `step.table`, the list,
    `step.counts[:1]`) blocks of tokens that are not kept are put back on the list, in place."""
    return Accepted._make((_binding or _native()).accept_path(tokens, parents, choices, cu_seqlens, cached_lens, block_size, table,
                                                              free_blocks, n_free))


def keep_path(caches, table, cu_seqlens, cached_lens, path) -> None:
    """Keys and values of the kept tokens to where a chain of tokens has them, in every cache of the list `caches` (k_cache and
    v_cache of all layers), in place.  `cached_lens` are the step's."""
    (_binding or _native()).keep_path(caches, table, cu_seqlens, cached_lens, path)
