"""Group norm with its activation on channels-last activations, forward and backward, on the GPU.

``pp_group_norm`` and ``pp_group_norm_backward`` mirror the C entry points (include/patconv.h);
``group_norm`` is the same as one differentiable operation.  Tensors are [N, C, H, W] in
``torch.channels_last`` order, float32, float16 or bfloat16, and may be a range of channels of a wider
channels-last tensor; gamma and beta are float32.  Every step runs in the library's kernels, and a
tensor that is elsewhere or in another order is rejected rather than copied or computed otherwise.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import _lib

ACTS = {"none": 0, "relu": 1, "silu": 2}
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
