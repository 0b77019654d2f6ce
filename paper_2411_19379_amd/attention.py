"""ctypes binding of the attention layers' operators (`include/attn_cache.h`): argument marshalling only.

    step = assign_blocks(block_size, total_tokens, cu_seqlens, cached_lens, table, free_blocks, n_free)   # once per step
    q = rope_append(q, k, v, step.positions, step.slots, rotary, k_cache, v_cache, copies=step.copies)    # once per layer
    out = attend(q, k_cache, v_cache, step.table, cu_seqlens, cached_lens)

All of it is enqueued on the current torch stream, nothing waits for the GPU, and lengths are read there; outputs and the
workspace are torch tensors.  There is no CPU fallback: loading raises if the library has not been built.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple, Optional

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
    # PyTorch owns device memory and streams here: its HIP runtime is the one this library has to bind to
    import torch  # noqa: F401

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


def _dtype_code(dtype) -> int:
    import torch

    code = {torch.float32: ATTN_DT_F32, torch.bfloat16: ATTN_DT_BF16, torch.float16: ATTN_DT_F16}.get(dtype)
    if code is None:
        raise ValueError(f"expected float32, bfloat16 or float16, got {dtype}")
    return code


def _tensor(name, t, shape, dtype, device):
    """A contiguous tensor of this shape (None: any extent) and type on `device`."""
    if t.dtype != dtype or t.dim() != len(shape) or t.device != device or not t.is_contiguous() \
            or any(want is not None and have != want for have, want in zip(t.shape, shape)):
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(name, t, shape, dtype, device):
    """[tokens, heads, head_dim] whose heads are contiguous; returns the address and the elements between tokens."""
    if t.dtype != dtype or t.device != device or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected a {dtype} tensor of shape {shape} on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    tokens, heads, dim = t.stride()
    row = shape[1] * shape[2]
    if (dim != 1 and shape[2] > 1) or (heads != shape[2] and shape[1] > 1):
        raise ValueError(f"{name}: the heads of a token must be contiguous, got strides {t.stride()}")
    return t.data_ptr(), (tokens if shape[0] > 1 else row)


def _device(t):
    import torch

    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"expected tensors on the current CUDA device, got {t.device}")
    return t.device


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
    import torch

    dev = _device(cu_seqlens)
    i32 = torch.int32
    batch = cu_seqlens.numel() - 1
    cu = _tensor("cu_seqlens", cu_seqlens, (batch + 1,), i32, dev)
    cached = _tensor("cached_lens", cached_lens, (batch,), i32, dev)
    tab = _tensor("table", table, (batch, None), i32, dev)
    free = _tensor("free_blocks", free_blocks, (None,), i32, dev)
    n = _tensor("n_free", n_free, (1,), i32, dev)
    shared = _tensor("shared_tail", shared_tail, (batch,), i32, dev) if shared_tail is not None else None
    out = table if in_place else torch.empty_like(table)
    slots = torch.empty((total_tokens,), dtype=torch.int64, device=dev)
    small = torch.empty((total_tokens + 4 * batch + 2,), dtype=i32, device=dev)
    positions, copies, counts = small[:total_tokens], small[total_tokens:-2].view(batch, 4), small[-2:]
    _check(load_library().attn_assign_blocks(
        batch, block_size, table.shape[1], total_tokens, cu, cached, shared, tab, out.data_ptr(), free, n,
        free_blocks.numel(), slots.data_ptr(), positions.data_ptr(), copies.data_ptr(), counts.data_ptr(),
        torch.cuda.current_stream(dev).cuda_stream))
    return Step(out, slots, positions, copies, counts)


def rotary_table(max_positions: int, rotary_dim: int, base: float = 10000.0, *, linear: float = 1.0,
                 by_parts: float = 1.0, trained_positions: int = 4096, slow_turns: float = 1.0, fast_turns: float = 32.0,
                 device="cuda"):
    """[max_positions, 2, rotary_dim / 2] fp32: cos and sin of position * base^(-2 i / rotary_dim), in 64 bits and rounded
    once.  For contexts longer than the `trained_positions`: `linear` divides every position by that factor; `by_parts` (the
    interpolation by parts of arXiv 2309.00071) divides by that factor the frequencies that turn fewer than `slow_turns` times over
    the trained positions, keeps those that turn more than `fast_turns` times, goes over linearly between, and scales cos and
    sin by 0.1 ln(by_parts) + 1."""
    import torch

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


def _cache_shape(k_cache, v_cache, n_q_heads, dtype, device):
    if k_cache.dim() != 4:
        raise ValueError(f"k_cache: expected [n_blocks, n_kv_heads, block_size, head_dim], got {tuple(k_cache.shape)}")
    n_blocks, n_kv, bs, d = k_cache.shape
    _tensor("k_cache", k_cache, (n_blocks, n_kv, bs, d), dtype, device)
    _tensor("v_cache", v_cache, (n_blocks, n_kv, bs, d), dtype, device)
    return n_blocks, AttnShape(n_q_heads, n_kv, d, bs, _dtype_code(dtype))


def rope_append(q, k, v, positions, slots, rotary, k_cache, v_cache, *, interleaved: bool = False, copies=None, q_out=None):
    """Rotary positions on q and k, k and v into the cache; returns the turned q [tokens, n_q_heads, head_dim].
    q, k and v may be parts of one projection's rows.  `rotary` is a `rotary_table` or None, `copies` comes from
    `assign_blocks` where sequences share their tails."""
    import torch

    dev, dtype = _device(q), q.dtype
    T, hq = q.shape[0], q.shape[1]
    n_blocks, shape = _cache_shape(k_cache, v_cache, hq, dtype, dev)
    d, hkv = shape.head_dim, shape.n_kv_heads
    qp, qs = _heads("q", q, (T, hq, d), dtype, dev)
    kp, ks = _heads("k", k, (T, hkv, d), dtype, dev)
    vp, vs = _heads("v", v, (T, hkv, d), dtype, dev)
    slot = _tensor("slots", slots, (T,), torch.int64, dev)
    pos = table = copy = None
    most = rot = batch = 0
    if rotary is not None:
        pos = _tensor("positions", positions, (T,), torch.int32, dev)
        table = _tensor("rotary", rotary, (None, 2, None), torch.float32, dev)
        most, rot = rotary.shape[0], 2 * rotary.shape[2]
    if copies is not None:
        copy, batch = _tensor("copies", copies, (None, 4), torch.int32, dev), copies.shape[0]
    if q_out is None:
        q_out = torch.empty((T, hq, d), dtype=dtype, device=dev)
    out = _tensor("q_out", q_out, (T, hq, d), dtype, dev)
    _check(load_library().attn_rope_append(
        ctypes.byref(shape), T, batch, n_blocks, qp, qs, kp, ks, vp, vs, pos, slot, table, most, rot, int(interleaved),
        copy, out, k_cache.data_ptr(), v_cache.data_ptr(), torch.cuda.current_stream(dev).cuda_stream))
    return q_out


def attend(q, k_cache, v_cache, table, cu_seqlens, cached_lens, *, scale: Optional[float] = None, window: int = 0,
           sinks: int = 0, max_new: int = 0, out=None, return_lse: bool = False):
    """Attention of the new tokens over the cache.  Returns out [tokens, n_q_heads, head_dim], with `return_lse` also the
    log of the sum of exponentials [tokens, n_q_heads].  `scale` is 1 / sqrt(head_dim) if not given; `max_new`, the largest
    number of new tokens of any sequence, picks the faster kernel (0: not known)."""
    import torch

    dev, dtype = _device(q), q.dtype
    T, hq = q.shape[0], q.shape[1]
    n_blocks, shape = _cache_shape(k_cache, v_cache, hq, dtype, dev)
    d = shape.head_dim
    batch = cu_seqlens.numel() - 1
    qp, qs = _heads("q", q, (T, hq, d), dtype, dev)
    tab = _tensor("table", table, (batch, None), torch.int32, dev)
    cu = _tensor("cu_seqlens", cu_seqlens, (batch + 1,), torch.int32, dev)
    cached = _tensor("cached_lens", cached_lens, (batch,), torch.int32, dev)
    if out is None:
        out = torch.empty((T, hq, d), dtype=dtype, device=dev)
    op, os_ = _heads("out", out, (T, hq, d), dtype, dev)
    lse = torch.empty((T, hq), dtype=torch.float32, device=dev) if return_lse else None
    need = attn_workspace_bytes(shape, batch, T, max_new)
    ws = torch.empty((need,), dtype=torch.uint8, device=dev) if need else None
    _check(load_library().attn_attend(
        ctypes.byref(shape), batch, T, n_blocks, table.shape[1], qp, qs, k_cache.data_ptr(), v_cache.data_ptr(), tab, cu,
        cached, 1.0 / math.sqrt(d) if scale is None else scale, window, sinks, max_new, op, os_,
        lse.data_ptr() if return_lse else None, ws.data_ptr() if need else None, need,
        torch.cuda.current_stream(dev).cuda_stream))
    return (out, lse) if return_lse else out
