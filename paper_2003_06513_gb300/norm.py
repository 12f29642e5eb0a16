"""Group norm with its activation on channels-last activations, forward and backward, on the GPU.

``pp_group_norm`` and ``pp_group_norm_backward`` mirror the C entry points (include/patconv.h);
``group_norm`` is the same as one differentiable operation.  Tensors are [N, C, H, W] in
``torch.channels_last`` order, float32, float16 or bfloat16, and may be a range of channels of a wider
channels-last tensor; gamma and beta are float32.  Every step runs in the library's kernels, and a
tensor that is elsewhere or in another order is rejected rather than copied or computed otherwise.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import Optional, Tuple

import torch

from . import _lib
from .api import _raw_stream

ACTS = {"none": 0, "relu": 1, "silu": 2}
_DT = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _strides(t: torch.Tensor) -> Optional[Tuple[int, int]]:
    """(elements between pixels, elements between samples) of a channels-last tensor, None of another."""
    n, c, h, w = t.shape
    sn, sc, sh, sw = t.stride()
    if c > 1 and sc != 1:
        return None
    if w > 1:
        pixel = sw
        if h > 1 and sh != w * sw:
            return None
    else:
        pixel = sh if h > 1 else c
    if pixel < c:
        return None
    return pixel, sn if n > 1 else 0


def _check(t: torch.Tensor, what: str) -> Tuple[int, int]:
    if not t.is_cuda or t.dtype not in _DT or t.dim() != 4:
        raise ValueError(f"{what} must be a 4-d CUDA float32, float16 or bfloat16 tensor")
    if t.numel() == 0:
        return t.shape[1], 0
    strides = _strides(t)
    if strides is None:
        raise ValueError(f"{what} must be channels last (strides {t.stride()} of {tuple(t.shape)})")
    return strides


def _address(t: Optional[torch.Tensor], count: int, x: torch.Tensor, what: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != count or not t.is_contiguous() or t.get_device() != x.get_device():
        raise ValueError(f"{what} must be {count} contiguous float32 values on the activations' device")
    return t.data_ptr()


def _on(x: torch.Tensor, stream):
    """The activations' device and, where one is given, the stream are current within."""
    stack = contextlib.ExitStack()
    if x.get_device() != torch.cuda.current_device():
        stack.enter_context(torch.cuda.device(x.get_device()))
    if stream is not None:
        stack.enter_context(torch.cuda.stream(stream))
    return stack


def _like(x: torch.Tensor, out: Optional[torch.Tensor], what: str) -> torch.Tensor:
    if out is None:
        return torch.empty(x.shape, dtype=x.dtype, device=x.device, memory_format=torch.channels_last)
    if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device \
            or not out.is_contiguous(memory_format=torch.channels_last):
        raise ValueError(f"{what} must be a dense channels-last tensor of x's shape, type and device")
    return out


def workspace_bytes(x_shape, groups: int, dtype=torch.float32, backward: bool = False) -> int:
    """Workspace of a call on activations of this shape and type (pp_group_norm_workspace_size)."""
    n, c, h, w = x_shape
    v = ctypes.c_size_t()
    _lib.check("pp_group_norm_workspace_size", _lib.load().pp_group_norm_workspace_size(
        _DT[dtype], n, h * w, c, groups, 1 if backward else 0, ctypes.byref(v)))
    return int(v.value)


def _workspace(x, groups, backward, workspace):
    need = workspace_bytes(x.shape, groups, x.dtype, backward)
    if workspace is None:
        workspace = torch.empty(max(16, need), dtype=torch.uint8, device=x.device)
    elif not workspace.is_contiguous() or workspace.get_device() != x.get_device():
        raise ValueError("workspace must be a contiguous CUDA tensor on x's device")
    return workspace, workspace.numel() * workspace.element_size()


def _act(act: str) -> int:
    if act not in ACTS:
        raise ValueError(f"act must be one of {', '.join(ACTS)}")
    return ACTS[act]


def pp_group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None,
                  bias: Optional[torch.Tensor] = None, eps: float = 1e-5, act: str = "none",
                  out: Optional[torch.Tensor] = None, stream=None, workspace: Optional[torch.Tensor] = None):
    """(y, mean, rstd): act(group_norm(x)), and the float32 [N, groups] that the backward pass needs."""
    pixel, sample = _check(x, "x")
    a, (n, c, h, w) = _act(act), x.shape
    if groups < 1 or c % groups:
        raise ValueError(f"{c} channels do not make {groups} groups")
    gamma, beta = _address(weight, c, x, "weight"), _address(bias, c, x, "bias")
    with _on(x, stream):
        y = _like(x, out, "out")
        stats = torch.empty((2, n, groups), dtype=torch.float32, device=x.device)
        mean, rstd = stats[0], stats[1]
        ws, ws_bytes = _workspace(x, groups, False, workspace)
        _lib.check("pp_group_norm", _lib.load().pp_group_norm(
            x.data_ptr(), pixel, sample, _DT[x.dtype], n, h * w, c, groups, gamma, beta, eps, a, y.data_ptr(),
            mean.data_ptr(), rstd.data_ptr(), ws.data_ptr(), ws_bytes, _raw_stream(stream, x.device)))
    return y, mean, rstd


def pp_group_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, groups: int,
                           weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                           act: str = "none", out: Optional[torch.Tensor] = None, stream=None,
                           workspace: Optional[torch.Tensor] = None):
    """(dx, dweight, dbias) from the gradient dy of y = act(group_norm(x)) and the forward pass's mean
    and rstd; weight and bias as they were there."""
    pixel, sample = _check(x, "x")
    dy_pixel, dy_sample = _check(dy, "dy")
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.device != x.device:
        raise ValueError("dy must have x's shape, type and device")
    a, (n, c, h, w) = _act(act), x.shape
    if groups < 1 or c % groups:
        raise ValueError(f"{c} channels do not make {groups} groups")
    gamma, beta = _address(weight, c, x, "weight"), _address(bias, c, x, "bias")
    mean_p, rstd_p = _address(mean, n * groups, x, "mean"), _address(rstd, n * groups, x, "rstd")
    with _on(x, stream):
        dx = _like(x, out, "out")
        sums = torch.empty((2, c), dtype=torch.float32, device=x.device)
        dgamma, dbeta = sums[0], sums[1]
        ws, ws_bytes = _workspace(x, groups, True, workspace)
        _lib.check("pp_group_norm_backward", _lib.load().pp_group_norm_backward(
            dy.data_ptr(), dy_pixel, dy_sample, x.data_ptr(), pixel, sample, _DT[x.dtype], n, h * w, c, groups,
            gamma, beta, mean_p, rstd_p, a, dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(), ws.data_ptr(),
            ws_bytes, _raw_stream(stream, x.device)))
    return dx, dgamma, dbeta


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
