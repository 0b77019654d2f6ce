"""Binding of the gated recurrent layers' operators (`include/gated_recurrence.h`): argument marshalling and the gradients' graph.

    h_t = a_t h_(t-1) + sqrt(1 - a_t^2) sigmoid(i_t) x_t,   a_t = exp(-sharpness softplus(decay) sigmoid(r_t)),   y_t = h_t

    out = gated_scan(x, r, i, decay, cu_seqlens, init_states=cached, ckpt=tokens)     # packed prompts; states for the prefix cache
    y = gated_step(x, r, i, decay, states)                                            # the next token of every sequence
    y, nodes = gated_step_tree(x, r, i, decay, states, cu_seqlens, parents)           # drafted trees (`attention.draft_tree`)
    keep_states(states, nodes, cu_seqlens, kept.path, kept.counts)                    # behind `attention.accept_path`

x, r, i and y are [tokens, channels] in float32, bfloat16 or float16; decay [channels] and all states are float32.  All of it is
enqueued on the current torch stream and nothing waits for the GPU.  There is no CPU fallback: loading raises if the library
has not been built.  `gated_scan` records a graph where an input requires grad; the others refuse such tensors, and all refuse those
with a tangent of forward-mode differentiation.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional

import torch  # owns device memory and streams; its HIP runtime is the one the library has to bind to

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libgated_recurrence.so")
_lib = None

REC_DT_F32, REC_DT_BF16, REC_DT_F16 = 0, 1, 2
REC_SAVED_EVERY = 8
REC_MOST_STRIDE = 1 << 22  # elements between tokens

_STATUS = {0: "REC_OK", -1: "REC_ERR_INVALID_ARG", -4: "REC_ERR_UNSUPPORTED_SHAPE", -5: "REC_ERR_WORKSPACE_TOO_SMALL",
           -6: "REC_ERR_MISALIGNED", -7: "REC_ERR_HIP"}


class RecError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_STATUS.get(code, code)}: {msg}")
        self.code = code
        self.status = _STATUS.get(code, str(code))


class RecShape(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("sharpness", ctypes.c_float)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libgated_recurrence.so (built by `python -m paper_2411_19379_amd.build`); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} is not built: run `python -m paper_2411_19379_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    shape = ctypes.POINTER(RecShape)
    inputs = [vp, i64, vp, i64, vp, i64, vp]  # x, r, i with their strides, decay
    lib.rec_workspace_bytes.restype = ctypes.c_int
    lib.rec_workspace_bytes.argtypes = [shape, i32, i64, i32, ctypes.POINTER(size)]
    lib.rec_scan.restype = ctypes.c_int
    lib.rec_scan.argtypes = [shape, i32, i64, *inputs, vp, vp, vp, i32, vp, i64, vp, vp, vp, vp, size, vp]
    lib.rec_scan_grads.restype = ctypes.c_int
    lib.rec_scan_grads.argtypes = [shape, i32, i64, *inputs, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, size, vp]
    lib.rec_step.restype = ctypes.c_int
    lib.rec_step.argtypes = [shape, i32, *inputs, vp, vp, i64, vp]
    lib.rec_step_tree.restype = ctypes.c_int
    lib.rec_step_tree.argtypes = [shape, i32, i64, *inputs, vp, vp, vp, vp, i64, vp, vp]
    lib.rec_keep_states.restype = ctypes.c_int
    lib.rec_keep_states.argtypes = [i32, i32, i64, vp, vp, vp, vp, vp, vp]
    lib.rec_last_error.restype = ctypes.c_char_p
    lib.rec_last_error.argtypes = []
    _lib = lib
    return lib


def rec_last_error() -> str:
    return load_library().rec_last_error().decode()


def rec_workspace_bytes(shape: RecShape, batch: int, total_tokens: int, grads: int = 0) -> int:
    n = ctypes.c_size_t()
    rc = load_library().rec_workspace_bytes(ctypes.byref(shape), batch, total_tokens, grads, ctypes.byref(n))
    if rc != 0:
        raise RecError(rc, rec_last_error())
    return n.value


_binding = None


def _native():
    """The compiled binding (csrc/rec_binding.cpp), which checks tensors and allocates outputs; raises if it is not built."""
    global _binding
    if _binding is None:
        load_library()
        try:
            from . import _rec_binding
        except ImportError as e:
            raise ImportError(f"the recurrence binding is not built or does not fit this torch ({e}): "
                              "run `python -m paper_2411_19379_amd.build`") from e
        _rec_binding.set_error_class(RecError)
        _binding = _rec_binding
    return _binding


class GatedScan(NamedTuple):
    """What `gated_scan` returns."""
    y: "torch.Tensor"                       # [tokens, channels]; rows of tokens of no sequence are not written
    final: "torch.Tensor"                   # [batch, channels] float32: the state behind every sequence
    ckpt_states: Optional["torch.Tensor"]   # [len(ckpt), channels] float32: the state behind each of the tokens; None without


class _Differentiable(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, r, i, decay, init_states, cu_seqlens, sharpness):
        y, final, _, saved = _native().scan(x, r, i, decay, cu_seqlens, sharpness, init_states, None, None, True)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x, r, i, decay, init_states, cu_seqlens, saved)
        ctx.sharpness = sharpness
        return y, final

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, d_final):
        x, r, i, decay, init_states, cu_seqlens, saved = ctx.saved_tensors
        _not_captured(x)
        if dy is None and d_final is None:
            return (None,) * 7
        if dy is not None and not _in_rows(dy):
            dy = dy.contiguous()  # an expanded gradient, as a sum's is, or rows further apart than the kernels take
        if d_final is not None:
            d_final = d_final.contiguous()
        grads = _native().scan_grads(x, r, i, decay, cu_seqlens, ctx.sharpness, init_states, saved, dy, d_final, init_states is not None)
        return (*(g if wanted else None for g, wanted in zip(grads, ctx.needs_input_grad)), None, None)


def _in_rows(t) -> bool:
    return t.stride(1) == 1 and t.shape[1] <= t.stride(0) <= REC_MOST_STRIDE or t.is_contiguous()


def _not_captured(x):
    if x.is_cuda and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("a graph of gradients is not captured: capture gated_scan under torch.no_grad() and gated_scan_grads")


def gated_scan(x, r, i, decay, cu_seqlens, *, sharpness: float = 8.0, init_states=None, ckpt=None, out=None) -> GatedScan:
    """The recurrence over packed sequences, sequence b being tokens cu_seqlens[b] .. cu_seqlens[b+1]-1 (int32, read on the GPU).
    `init_states` [batch, channels]: what sequences resume from, zeros if not given.  `ckpt` [any] int32: packed tokens behind
    which the state is wanted.  x, r and i may be parts of one projection's rows.

    Where an input requires grad the call can be differentiated once with respect to x, r, i, decay and init_states; there
    are no gradients through `ckpt`, and none into a given `out`."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, r, i, decay, init_states)):
        if ckpt is not None or out is not None:
            raise ValueError("ckpt and out are not differentiable: call under torch.no_grad(), or detach")
        _not_captured(x)
        return GatedScan(*_Differentiable.apply(x, r, i, decay, init_states, cu_seqlens, sharpness), None)
    if out is not None and out.requires_grad and torch.is_grad_enabled():
        raise ValueError("out requires grad: call under torch.no_grad(), or detach")
    return GatedScan(*(_binding or _native()).scan(x, r, i, decay, cu_seqlens, sharpness, init_states, ckpt, out, False)[:3])


class GatedGrads(NamedTuple):
    """What `gated_scan_grads` returns: x, r and i in their type, the others float32."""
    x: "torch.Tensor"
    r: "torch.Tensor"
    i: "torch.Tensor"
    decay: "torch.Tensor"
    init_states: "torch.Tensor"


def gated_scan_grads(dy, d_final, x, r, i, decay, cu_seqlens, *, sharpness: float = 8.0, init_states=None) -> GatedGrads:
    """The gradients of `gated_scan` without a recorded graph, for steps that are captured: from those of y and of the final states
    (None: zeros).  The states are computed again.  Tokens of no sequence get zeros."""
    with torch.no_grad():
        return GatedGrads(*(_binding or _native()).scan_grads(x, r, i, decay, cu_seqlens, sharpness, init_states, None, dy, d_final, True))


def gated_step(x, r, i, decay, states, *, sharpness: float = 8.0, out=None):
    """One token of every sequence: row b of x, r and i with row b of `states` [batch, channels], which is replaced.  Returns y."""
    return (_binding or _native()).step(x, r, i, decay, states, sharpness, out)


def gated_step_tree(x, r, i, decay, states, cu_seqlens, parents, *, sharpness: float = 8.0, out=None):
    """Trees of new tokens: each continues its parent (`parents` [tokens] int32, the index in its sequence; -1: the sequence's row
    of `states`, which stays).  Returns y and the state behind every token [tokens, channels]."""
    return (_binding or _native()).step_tree(x, r, i, decay, states, cu_seqlens, parents, sharpness, out)


def keep_states(states, node_states, cu_seqlens, path, counts) -> None:
    """`states` of the last kept token of every sequence, in place; path and counts as `attention.accept_path` returns them."""
    (_binding or _native()).keep_states(states, node_states, cu_seqlens, path, counts)
