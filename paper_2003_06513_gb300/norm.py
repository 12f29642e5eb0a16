"""Group norm with its activation, and block norm, on channels-last activations, forward and backward, on the GPU.

``pp_group_norm`` and ``pp_group_norm_backward`` mirror the C entry points (include/patconv.h);
``group_norm`` is the same as one differentiable operation.  ``pp_block_norm``, ``pp_block_norm_backward`` and
``block_norm`` are how a residual block joins its stream: the norm of the block's output, times gate and residual scale,
added to the stream, and the stream's norm with its activation, which the next block reads.  Tensors are [N, C, H, W] in
``torch.channels_last`` order, float32, float16 or bfloat16, and may be a range of channels of a wider
channels-last tensor; gamma and beta are float32.  Every step runs in the library's kernels, and a
tensor that is elsewhere or in another order is rejected rather than copied or computed otherwise.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple

import torch

from . import _lib

ACTS = {"none": 0, "relu": 1, "silu": 2}
NORMS = {"none": 0, "rms": 1, "layer": 2}
_DT = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _strides(t: torch.Tensor) -> Optional[Tuple[int, int]]:
    """(elements between pixels, elements between samples) of a channels-last tensor, None of another."""
    return _lib.binding().layout(t)


def workspace_bytes(x_shape, groups: int, dtype=torch.float32, backward: bool = False) -> int:
    """Workspace of a call on activations of this shape and type (pp_group_norm_workspace_size)."""
    n, c, h, w = x_shape
    v = ctypes.c_size_t()
    _lib.check("pp_group_norm_workspace_size", _lib.load().pp_group_norm_workspace_size(
        _DT[dtype], n, h * w, c, groups, 1 if backward else 0, ctypes.byref(v)))
    return int(v.value)


PLAN_KEYS = ("path", "channels", "columns", "pixels", "held", "cluster", "ctas", "sets")


def plan(x_shape, groups: int, dtype=torch.float32, backward: bool = False, align: int = 16) -> dict:
    """How a call on activations of this shape and type runs (pp_group_norm_plan): ``path`` 2 resident, 1
    streamed.  ``align``: the largest power of two that divides all addresses and strides in bytes."""
    n, c, h, w = x_shape
    info = (ctypes.c_int64 * len(PLAN_KEYS))()
    _lib.check("pp_group_norm_plan", _lib.load().pp_group_norm_plan(
        _DT[dtype], n, h * w, c, groups, 1 if backward else 0, align, info, len(PLAN_KEYS)))
    return dict(zip(PLAN_KEYS, (int(v) for v in info)))


def _act(act: str) -> int:
    if act not in ACTS:
        raise ValueError(f"act must be one of {', '.join(ACTS)}")
    return ACTS[act]


def _done(fn: str, result):
    if type(result) is int:
        raise _lib.PatconvError(fn, result)
    return result


def pp_group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None,
                  bias: Optional[torch.Tensor] = None, eps: float = 1e-5, act: str = "none",
                  out: Optional[torch.Tensor] = None, stream=None, workspace: Optional[torch.Tensor] = None):
    """(y, mean, rstd): act(group_norm(x)), and the float32 [N, groups] that the backward pass needs."""
    return _done("pp_group_norm", _lib.binding().group_norm(
        x, groups, weight, bias, eps, _act(act), out, None if stream is None else stream.cuda_stream, workspace))


def pp_group_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, groups: int,
                           weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                           act: str = "none", out: Optional[torch.Tensor] = None, stream=None,
                           workspace: Optional[torch.Tensor] = None):
    """(dx, dweight, dbias) from the gradient dy of y = act(group_norm(x)) and the forward pass's mean
    and rstd; weight and bias as they were there."""
    return _done("pp_group_norm_backward", _lib.binding().group_norm_backward(
        dy, x, mean, rstd, groups, weight, bias, _act(act), out, None if stream is None else stream.cuda_stream, workspace))


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act):
        y, mean, rstd = pp_group_norm(x, groups, weight, bias, eps, act)
        ctx.save_for_backward(x, weight, bias, mean, rstd)
        ctx.groups, ctx.act = groups, act
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, mean, rstd = ctx.saved_tensors
        if _strides(dy) is None:        # autograd hands over whatever order the next operation left
            dy = dy.contiguous(memory_format=torch.channels_last)
        dx, dweight, dbias = pp_group_norm_backward(dy, x, mean, rstd, ctx.groups, weight, bias, ctx.act)
        return (dx if ctx.needs_input_grad[0] else None, dweight if ctx.needs_input_grad[1] else None,
                dbias if ctx.needs_input_grad[2] else None, None, None, None)


def group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None,
               bias: Optional[torch.Tensor] = None, eps: float = 1e-5, act: str = "none") -> torch.Tensor:
    """act(group_norm(x)) as one differentiable operation, on the current stream."""
    return _GroupNorm.apply(x, weight, bias, groups, eps, act)


# ------------------------------------------------------------------------------------- block norm

def _norm(kind: str, what: str) -> int:
    if kind not in NORMS:
        raise ValueError(f"{what} must be one of {', '.join(NORMS)}")
    return NORMS[kind]


def block_workspace_bytes(x_shape) -> int:
    """Workspace of a backward pass of block norm on a stream of this shape (pp_block_norm_workspace_size)."""
    n, c, h, w = x_shape
    v = ctypes.c_size_t()
    _lib.check("pp_block_norm_workspace_size", _lib.load().pp_block_norm_workspace_size(n, h * w, c, ctypes.byref(v)))
    return int(v.value)


class BlockGrads(NamedTuple):
    """Gradients of a block norm, None where the argument was; those of the parameters are float32."""
    dx: torch.Tensor
    dblock: Optional[torch.Tensor]
    dpost_weight: Optional[torch.Tensor]
    dpost_bias: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dweight: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]


def pp_block_norm(x: torch.Tensor, block: Optional[torch.Tensor], post: str = "rms", post_weight: Optional[torch.Tensor] = None,
                  post_bias: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, pre: str = "rms", weight: Optional[torch.Tensor] = None,
                  bias: Optional[torch.Tensor] = None, act: str = "none", eps: float = 1e-5, out=(None, None), stream=None):
    """(h, y): h = x + scale * gate * norm_post(block), the new residual stream, and y = act(norm_pre(h)), over each
    pixel's channels.

    ``x``           the stream, float32 or of the block's type;
    ``block``       the block's output, or None: then h is x, and post must be "none";
    ``post, pre``   "rms" (by the root of the mean square), "layer" (without the mean) or "none" (pre: y is None);
    ``post_weight, post_bias, scale, weight, bias``  float32 [C], ``gate`` float32 [N, C]; each may be None;
    ``out``         (h, y) to write to, or None: h may be x, and y the block's output."""
    return _done("pp_block_norm", _lib.binding().block_norm(
        x, block, _norm(post, "post"), post_weight, post_bias, scale, gate, _norm(pre, "pre"), weight, bias, _act(act), eps,
        out[0], out[1], None if stream is None else stream.cuda_stream))


def pp_block_norm_backward(dh: Optional[torch.Tensor], dy: Optional[torch.Tensor], h: torch.Tensor,
                           block: Optional[torch.Tensor], post: str = "rms", post_weight: Optional[torch.Tensor] = None,
                           post_bias: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                           gate: Optional[torch.Tensor] = None, pre: str = "rms", weight: Optional[torch.Tensor] = None,
                           bias: Optional[torch.Tensor] = None, act: str = "none", eps: float = 1e-5, out=(None, None), stream=None,
                           workspace: Optional[torch.Tensor] = None) -> BlockGrads:
    """The gradients from those of h and y (None: zero); h is the forward pass's, the other arguments as they were there.
    ``out``: (dx, dblock) to write to, or None: dx may be dh, and dblock dy."""
    return BlockGrads(*_done("pp_block_norm_backward", _lib.binding().block_norm_backward(
        dh, dy, h, block, _norm(post, "post"), post_weight, post_bias, scale, gate, _norm(pre, "pre"), weight, bias, _act(act), eps,
        out[0], out[1], None if stream is None else stream.cuda_stream, workspace)))


def _ordered(d: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A gradient as autograd hands it over, in channels-last order."""
    return d if d is None or _strides(d) is not None else d.contiguous(memory_format=torch.channels_last)


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, block, post_weight, post_bias, scale, gate, weight, bias, post, pre, act, eps):
        h, y = pp_block_norm(x, block, post, post_weight, post_bias, scale, gate, pre, weight, bias, act, eps)
        ctx.set_materialize_grads(False)
        ctx.kinds = post, pre, act, eps
        ctx.save_for_backward(h if block is not None else x, block, post_weight, post_bias, scale, gate, weight, bias)
        return (h, y) if block is not None else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        h, block, post_weight, post_bias, scale, gate, weight, bias = ctx.saved_tensors
        post, pre, act, eps = ctx.kinds
        dh, dy = grads if block is not None else (None, grads[0])
        if dh is None and dy is None:
            return (None,) * 12
        g = pp_block_norm_backward(_ordered(dh), _ordered(dy), h, block, post, post_weight, post_bias, scale, gate, pre, weight,
                                   bias, act, eps)
        wanted = (g.dx, g.dblock, g.dpost_weight, g.dpost_bias, g.dscale, g.dgate, g.dweight, g.dbias)
        return tuple(d if need else None for d, need in zip(wanted, ctx.needs_input_grad)) + (None,) * 4


def block_norm(x: torch.Tensor, block: Optional[torch.Tensor], post: str = "rms", post_weight: Optional[torch.Tensor] = None,
               post_bias: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
               gate: Optional[torch.Tensor] = None, pre: str = "rms", weight: Optional[torch.Tensor] = None,
               bias: Optional[torch.Tensor] = None, act: str = "none", eps: float = 1e-5):
    """(h, y) of ``pp_block_norm`` as one differentiable operation, on the current stream.  Captured into a graph, its leaves
    are such that no living eager graph was built from."""
    got = _BlockNorm.apply(x, block, post_weight, post_bias, scale, gate, weight, bias, post, pre, act, eps)
    return got if block is not None else (x, got)
