"""ctypes binding of the attention layers' operators (`include/attn_cache.h`): argument marshalling only.

    step = assign_blocks(block_size, total_tokens, cu_seqlens, cached_lens, table, free_blocks, n_free)   # once per step
    q = rope_append(q, k, v, step.positions, step.slots, rotary, k_cache, v_cache, copies=step.copies)    # once per layer
    out = attend(q, k_cache, v_cache, step.table, cu_seqlens, cached_lens)

All of it is enqueued on the current torch stream, nothing waits for the GPU, and lengths are read there; outputs and the
workspace are torch tensors.  There is no CPU fallback: loading raises if the library has not been built.
"""
from __future__ import annotations

import ctypes
import functools
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


# A decode step of one layer is a few microseconds of GPU work and each line here costs a tenth of one: what follows from sizes
# alone is kept, and tensors are checked in one expression each.
_DTYPES = {torch.float32: ATTN_DT_F32, torch.bfloat16: ATTN_DT_BF16, torch.float16: ATTN_DT_F16}
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32
# the raw handle of a GPU's current stream, without the object that torch.cuda.current_stream makes where there is a way
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


@functools.lru_cache(maxsize=256)
def _shape_of(n_q_heads, n_kv_heads, head_dim, block_size, dtype):
    """The address of the shape."""
    if dtype not in _DTYPES:
        raise ValueError(f"expected float32, bfloat16 or float16, got {dtype}")
    return ctypes.byref(AttnShape(n_q_heads, n_kv_heads, head_dim, block_size, _DTYPES[dtype]))


@functools.lru_cache(maxsize=4096)
def _workspace_of(n_q_heads, n_kv_heads, head_dim, block_size, dtype, batch, total_tokens, max_new):
    shape = AttnShape(n_q_heads, n_kv_heads, head_dim, block_size, _DTYPES[dtype])
    return attn_workspace_bytes(shape, batch, total_tokens, max_new)


def _refuse(name, t, shape, dtype, index):
    raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{index}, "
                     f"got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _ints(name, t, n, index):
    """The address of n contiguous int32 values on GPU `index` (n None: any number)."""
    if t.dtype is not _I32 or t.get_device() != index or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n):
        _refuse(name, t, (n,), _I32, index)
    return t.data_ptr()


def _rows(name, t, n, index):
    """The address and the width of n contiguous rows of int32 values."""
    have = t.shape
    if t.dtype is not _I32 or t.get_device() != index or len(have) != 2 or have[0] != n or not t.is_contiguous():
        _refuse(name, t, (n, "any"), _I32, index)
    return t.data_ptr(), have[1]


def _tensor(name, t, shape, dtype, index):
    """The address of a contiguous tensor."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        _refuse(name, t, shape, dtype, index)
    return t.data_ptr()


def _heads(name, t, shape, dtype, index):
    """[tokens, heads, head_dim] whose heads are contiguous; returns the address and the elements between tokens."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        _refuse(name, t, shape, dtype, index)
    tokens, heads, dim = t.stride()
    if (dim != 1 and shape[2] > 1) or (heads != shape[2] and shape[1] > 1):
        raise ValueError(f"{name}: the heads of a token must be contiguous, got strides {t.stride()}")
    return t.data_ptr(), (tokens if shape[0] > 1 else shape[1] * shape[2])


def _device(t):
    """The index of the current GPU, which the tensor has to be on."""
    index = t.get_device()
    if index < 0 or index != torch.cuda.current_device():
        raise ValueError(f"expected tensors on the current CUDA device, got {t.device}")
    return index


class Step(NamedTuple):
    """What `assign_blocks` returns; device tensors."""
    table: "torch.Tensor"      # [batch, max_blocks] int32
    slots: "torch.Tensor"      # [total_tokens] int64, -1: no block
    positions: "torch.Tensor"  # [total_tokens] int32
    copies: "torch.Tensor"     # [batch, 4] int32: from block, to block, rows, 0
    counts: "torch.Tensor"     # [2] int32: free blocks left, blocks missing


def assign_blocks(block_size: int, total_tokens: int, cu_seqlens, cached_lens, table, free_blocks, n_free,
                  shared_tail=None, in_place: bool = False) -> Step:
    """Blocks, slots and positions of the new tokens of a batch.  `n_free` is a device int32 tensor of one value; the
    next step's is `counts[:1]` of this one.  `in_place` extends the rows of `table`, else they are written to a new one."""
    dev = _device(cu_seqlens)
    batch = cu_seqlens.numel() - 1
    tab, width = _rows("table", table, batch, dev)
    out = table if in_place else torch.empty_like(table)
    slots = torch.empty((total_tokens,), dtype=_I64, device=table.device)
    positions, copies, counts = table.new_empty((total_tokens,)), table.new_empty((batch, 4)), table.new_empty((2,))
    _check(load_library().attn_assign_blocks(
        batch, block_size, width, total_tokens, _ints("cu_seqlens", cu_seqlens, batch + 1, dev),
        _ints("cached_lens", cached_lens, batch, dev),
        None if shared_tail is None else _ints("shared_tail", shared_tail, batch, dev), tab, out.data_ptr(),
        _ints("free_blocks", free_blocks, None, dev), _ints("n_free", n_free, 1, dev), free_blocks.numel(), slots.data_ptr(),
        positions.data_ptr(), copies.data_ptr(), counts.data_ptr(), _stream(dev)))
    return Step(out, slots, positions, copies, counts)


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


def _caches(k_cache, v_cache, dtype, index):
    """The caches' extents and addresses."""
    extents = k_cache.shape
    if len(extents) != 4:
        raise ValueError(f"k_cache: expected [n_blocks, n_kv_heads, block_size, head_dim], got {tuple(extents)}")
    return extents, _tensor("k_cache", k_cache, extents, dtype, index), _tensor("v_cache", v_cache, extents, dtype, index)


def rope_append(q, k, v, positions, slots, rotary, k_cache, v_cache, *, interleaved: bool = False, copies=None, q_out=None):
    """Rotary positions on q and k, k and v into the cache; returns the turned q [tokens, n_q_heads, head_dim].
    q, k and v may be parts of one projection's rows.  `rotary` is a `rotary_table` or None, `copies` comes from
    `assign_blocks` where sequences share their tails."""
    dev, dtype = _device(q), q.dtype
    T, hq = q.shape[:2]
    (n_blocks, hkv, bs, d), k_to, v_to = _caches(k_cache, v_cache, dtype, dev)
    shape = _shape_of(hq, hkv, d, bs, dtype)
    q_shape, kv_shape = (T, hq, d), (T, hkv, d)
    qp, qs = _heads("q", q, q_shape, dtype, dev)
    kp, ks = _heads("k", k, kv_shape, dtype, dev)
    vp, vs = _heads("v", v, kv_shape, dtype, dev)
    pos = table = copy = None
    most = rot = batch = 0
    if rotary is not None:
        pos = _ints("positions", positions, T, dev)
        if rotary.dim() != 3 or rotary.shape[1] != 2:
            raise ValueError(f"rotary: expected [positions, 2, rotary_dim / 2], got {tuple(rotary.shape)}")
        most, _, rot = rotary.shape
        table, rot = _tensor("rotary", rotary, (most, 2, rot), _F32, dev), 2 * rot
    if copies is not None:
        batch = copies.shape[0]
        copy = _tensor("copies", copies, (batch, 4), _I32, dev)
    if q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    _check(load_library().attn_rope_append(
        shape, T, batch, n_blocks, qp, qs, kp, ks, vp, vs, pos, _tensor("slots", slots, (T,), _I64, dev), table, most, rot,
        int(interleaved), copy, _tensor("q_out", q_out, q_shape, dtype, dev), k_to, v_to, _stream(dev)))
    return q_out


def attend(q, k_cache, v_cache, table, cu_seqlens, cached_lens, *, scale: Optional[float] = None, window: int = 0,
           sinks: int = 0, max_new: int = 0, out=None, return_lse: bool = False):
    """Attention of the new tokens over the cache.  Returns out [tokens, n_q_heads, head_dim], with `return_lse` also the
    log of the sum of exponentials [tokens, n_q_heads].  `scale` is 1 / sqrt(head_dim) if not given; `max_new`, the largest
    number of new tokens of any sequence, picks the faster kernel (0: not known)."""
    dev, dtype = _device(q), q.dtype
    T, hq = q.shape[:2]
    (n_blocks, hkv, bs, d), kp, vp = _caches(k_cache, v_cache, dtype, dev)
    shape = _shape_of(hq, hkv, d, bs, dtype)
    batch = cu_seqlens.numel() - 1
    q_shape = (T, hq, d)
    qp, qs = _heads("q", q, q_shape, dtype, dev)
    tab, width = _rows("table", table, batch, dev)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    op, os_ = _heads("out", out, q_shape, dtype, dev)
    lse = torch.empty((T, hq), dtype=_F32, device=q.device) if return_lse else None
    need = _workspace_of(hq, hkv, d, bs, dtype, batch, T, max_new)
    ws = torch.empty((need,), dtype=torch.uint8, device=q.device) if need else None
    _check(load_library().attn_attend(
        shape, batch, T, n_blocks, width, qp, qs, kp, vp, tab, _ints("cu_seqlens", cu_seqlens, batch + 1, dev),
        _ints("cached_lens", cached_lens, batch, dev), 1.0 / math.sqrt(d) if scale is None else scale, window, sinks, max_new,
        op, os_, lse.data_ptr() if return_lse else None, ws.data_ptr() if need else None, need, _stream(dev)))
    return (out, lse) if return_lse else out
