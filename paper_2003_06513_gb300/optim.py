"""The optimiser of masked retraining: gradient norm and AdamW over many tensors in one launch each.

``AdamW`` holds the handle of a list of parameters (include/patconv.h, pp_tensors_*), its tables on
the device and the two moments, in fp32 or in 8 bits.  Weights given with their tap masks
(``taps_of``) keep their pattern and connectivity: the step leaves pruned taps alone, whatever their
gradient holds, so the hooks of ``admm.masked_retraining_hook`` are not needed beside it.
``GradNorm`` gives the norm of a list of gradients and the factor that clips them, both on the
device; ``AdamW.grad_norm`` is the same for its own gradients.  Nothing here waits for the GPU but
the constructors, which copy a table to it.

    opt = AdamW(weights, lr=1e-3, weight_decay=0.05, state_bits=8, taps=[taps_of(w) for w in weights])
    norm, scale = opt.grad_norm(grads, max_norm=1.0)
    opt.step(grads, grad_scale=scale)
"""
from __future__ import annotations

import contextlib
import ctypes
import math
from typing import Optional, Sequence, Union

import torch

from . import _lib
from .api import _raw_stream, _stream_ptr

PP_F32, PP_F16, PP_BF16 = 0, 1, 2
_DT = {torch.float32: PP_F32, torch.float16: PP_F16, torch.bfloat16: PP_BF16}
_COUNT, _TABLE_BYTES, _STATE_ELEMENTS, _STATE_OFFSET = 0, 1, 2, 16
STATE_BLOCK = 256


def taps_of(weight: torch.Tensor) -> torch.Tensor:
    """Tap masks of a pruned weight [Cout, Cin/groups, 3, 3]: int16 [Cout * Cin/groups], bit t set where
    raster tap t is not zero now; 0 for a kernel that is pruned away."""
    if weight.dim() != 4 or tuple(weight.shape[2:]) != (3, 3):
        raise ValueError("weight must be [Cout, Cin/groups, 3, 3]")
    bits = torch.tensor([1 << t for t in range(9)], dtype=torch.int32, device=weight.device)
    return ((weight.detach().reshape(-1, 9) != 0).int() * bits).sum(1).to(torch.int16)


def _per_tensor(value, n: int, what: str) -> list:
    values = list(value) if isinstance(value, (list, tuple)) else [value] * n
    if len(values) != n:
        raise ValueError(f"{what}: {len(values)} values for {n} tensors")
    return values


def _dense(t: torch.Tensor) -> bool:
    """Whether the tensor's elements fill one stretch of memory, in whatever order of dimensions."""
    if t.numel() == 0:
        return True
    step = 1
    for stride, size in sorted((s, k) for s, k in zip(t.stride(), t.shape) if k != 1):
        if stride != step:
            return False
        step *= size
    return True


def _contiguous_strides(shape) -> tuple:
    out, step = [], 1
    for k in reversed(shape):
        out.append(step)
        step *= max(1, k)
    return tuple(reversed(out))


class _Tensors:
    """A pp_tensors handle with its table on the device."""

    def __init__(self, shapes, strides, grad_dtypes, taps, device, params=None, copies=None, decay=None, stream=None):
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError("the tensors must live in CUDA device memory")
        index = device.index if device.index is not None else torch.cuda.current_device()
        self._h = None
        self._device, self._index = torch.device("cuda", index), index
        n = len(shapes)
        sizes = [math.prod(s) for s in shapes]
        dtypes = _per_tensor(grad_dtypes, n, "grad_dtypes")
        if any(d not in _DT for d in dtypes):
            raise ValueError("gradients must be float32, float16 or bfloat16")
        taps = _per_tensor(taps, n, "taps")
        for t, shape, size in zip(taps, shapes, sizes):
            if t is None:
                continue
            if len(shape) != 4 or tuple(shape[2:]) != (3, 3) or 9 * t.numel() != size:
                raise ValueError("taps go with a [Cout, Cin/groups, 3, 3] tensor, one mask a kernel")
            if t.dtype != torch.int16 or not t.is_contiguous() or t.get_device() != index:
                raise ValueError("taps must be contiguous int16 tensors on the tensors' device")
        # the memory that the table has addresses of: the tensors may be given other memory, and free this
        self._keep_alive = [t.detach() for ts in (taps, params, copies) for t in ts or [] if t is not None]
        copy_dtype = next((_DT[c.dtype] for c in copies or [] if c is not None), PP_F16)

        def addresses(tensors):
            return (ctypes.c_void_p * max(1, n))(*[t.data_ptr() if t is not None else None for t in tensors])

        h = ctypes.c_void_p()
        lib = _lib.load()
        _lib.check("pp_tensors_create", lib.pp_tensors_create(
            n, (ctypes.c_int64 * max(1, n))(*sizes), (ctypes.c_int * max(1, n))(*[_DT[d] for d in dtypes]),
            addresses(taps), addresses(params) if params is not None else None,
            addresses(copies) if copies is not None else None, copy_dtype,
            (ctypes.c_float * max(1, n))(*decay) if decay is not None else None, ctypes.byref(h)))
        self._h = h
        self.native = _lib.binding()
        self.list = self.native.tensors(h.value, index, [(tuple(shape), tuple(stride), _DT[d])
                                                         for shape, stride, d in zip(shapes, strides, dtypes)],
                                        [(t, i) for ts in (params, copies) for i, t in enumerate(ts or []) if t is not None])
        self._home = _raw_stream(stream, self._device)      # the stream that what is allocated here belongs to
        with torch.cuda.device(index), self._on(stream):
            self._table = torch.empty(self.query(_TABLE_BYTES), dtype=torch.uint8, device=self._device)
            _lib.check("pp_tensors_bind", lib.pp_tensors_bind(h, ctypes.c_void_p(self._table.data_ptr()),
                                                              self._table.numel(), _stream_ptr(stream, self._device)))
            self.settle()

    def query(self, key: int) -> int:
        v = ctypes.c_int64()
        _lib.check("pp_tensors_query", _lib.load().pp_tensors_query(self._h, key, ctypes.byref(v)))
        return int(v.value)

    def settle(self) -> None:
        """Waits for what the constructor has put on the current stream, unless that is being captured: calls on any
        stream may follow."""
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()

    def _on(self, stream):
        return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()

    def used(self, tensors, stream) -> None:
        """Keeps the memory of the table and of ``tensors`` from another use before a call's stream is done with
        them, where that is not the stream they belong to."""
        if _raw_stream(stream, self._device) != self._home:
            on = stream if stream is not None else torch.cuda.current_stream(self._device)
            for t in (self._table, *tensors):
                if t is not None:
                    t.record_stream(on)

    def norm(self, grads, max_norm, out, stream):
        self.used((), stream)
        got = self.native.grad_norm(self.list, grads, max_norm, out, None if stream is None else stream.cuda_stream)
        if type(got) is int:
            raise _lib.PatconvError("pp_grad_norm", got)
        return got

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            try:
                _lib.load().pp_tensors_destroy(h)
            except Exception:
                pass


class GradNorm:
    """Norm and clip factor of a list of gradients of the given shapes (pp_grad_norm); with ``taps``
    (a list, None where a tensor is not masked) of the kept elements alone.  Order calls on one object."""

    def __init__(self, shapes: Sequence, grad_dtypes: Union[torch.dtype, Sequence] = torch.float32,
                 taps: Optional[Sequence] = None, device="cuda", stream=None):
        shapes = [tuple(s) for s in shapes]
        self._t = _Tensors(shapes, [_contiguous_strides(s) for s in shapes], grad_dtypes, taps, device, stream=stream)

    def __call__(self, grads: Sequence, max_norm: float = math.inf, out: Optional[torch.Tensor] = None, stream=None):
        """(norm, scale): the norm of all gradients, and min(1, max_norm / (norm + 1e-6)), one float32
        each on the device.  ``grads``: contiguous tensors, None where there is no gradient."""
        return self._t.norm(grads, max_norm, out, stream)


class AdamW:
    """AdamW over a list of float32 CUDA parameters, updated in place (pp_adamw_step).

    ``params``        dense tensors of any shape; contiguous where they have a mask;
    ``weight_decay``  one value, or one a tensor;
    ``state_bits``    32, or 8: moments in float8_e4m3fn with a power of two for every 256 elements;
    ``taps``          None, or per tensor None or its tap masks (``taps_of``);
    ``grad_dtypes``   one type, or one a tensor (float32, float16, bfloat16);
    ``copies``        None, or per tensor None or a float16 / bfloat16 tensor of the same shape and
                      order that each step writes the rounded parameters to;
    ``seed``          of the 8-bit states' rounding;
    ``state``         what ``state_dict`` gave: its tensors become this object's own.

    Parameters and copies share no memory: one that is used twice is given once, with the sum of its gradients.
    Parameters, copies and masks keep their memory while the object is used: ``step`` refuses a parameter or copy that
    was given other memory (``p.data = ...``, a module's move to another type or order); masks are read where they were.
    ``m`` and ``v`` (and ``m_scale``, ``v_scale``) hold all tensors' moments one after the other, each
    from a multiple of 256 elements on; ``state_of`` gives one tensor's."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.01, state_bits: int = 32,
                 taps: Optional[Sequence] = None, grad_dtypes: Union[torch.dtype, Sequence] = torch.float32,
                 copies: Optional[Sequence] = None, seed: int = 0, state: Optional[dict] = None, stream=None):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        n, device = len(self.params), self.params[0].device
        taps = _per_tensor(taps, n, "taps")
        for p, t in zip(self.params, taps):
            if not p.is_cuda or p.dtype != torch.float32 or p.device != device or not _dense(p):
                raise ValueError("parameters must be dense float32 tensors on one CUDA device")
            if t is not None and not p.is_contiguous():
                raise ValueError("a parameter with a mask must be contiguous")
        if copies is not None:
            copies = _per_tensor(copies, n, "copies")
            dtypes = {c.dtype for c in copies if c is not None}
            if len(dtypes) > 1 or not dtypes <= {torch.float16, torch.bfloat16}:
                raise ValueError("copies must be all float16 or all bfloat16")
            for p, c in zip(self.params, copies):
                if c is not None and (c.shape != p.shape or c.stride() != p.stride() or c.device != device):
                    raise ValueError("a copy must have its parameter's shape, strides and device")
        self._written = self.params + [c for c in copies or [] if c is not None]
        self.lr, self.betas, self.eps, self.seed, self.state_bits = lr, tuple(betas), eps, int(seed) & 0xFFFFFFFF, state_bits
        self.steps = 0
        self._t = _Tensors([p.shape for p in self.params], [p.stride() for p in self.params], grad_dtypes, taps, device,
                           self.params, copies, [float(w) for w in _per_tensor(weight_decay, n, "weight_decay")], stream)
        count = self._t.query(_STATE_ELEMENTS)
        blocks = count // STATE_BLOCK
        dtype = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        self.m_scale = self.v_scale = None
        if state is None:
            with torch.cuda.device(device), self._t._on(stream):
                self.m, self.v = (torch.zeros(count * (4 if state_bits == 32 else 1), dtype=torch.uint8,
                                              device=device).view(dtype) for _ in range(2))
                if state_bits == 8:
                    self.m_scale, self.v_scale = (torch.ones(blocks, device=device) for _ in range(2))
                self._t.settle()
        else:
            wanted = {"m": (dtype, count), "v": (dtype, count)}
            if state_bits == 8:
                wanted |= {"m_scale": (torch.float32, blocks), "v_scale": (torch.float32, blocks)}
            for name, (dt, size) in wanted.items():
                t = state[name]
                if t.dtype != dt or t.numel() != size or not t.is_contiguous() or t.device != device:
                    raise ValueError(f"state {name} must be {size} contiguous {dt} values on {device}")
                setattr(self, name, t)
            self.steps = int(state["step"])
            if "missed" in state:
                self._t.native.missed(self._t.list, list(state["missed"]))

    def state_dict(self) -> dict:
        """The moments, the step count and, per tensor, the steps at which it had no gradient; the tensors are this
        object's own, not copies."""
        d = {"m": self.m, "v": self.v, "step": self.steps, "missed": self._t.native.missed(self._t.list, None)}
        if self.state_bits == 8:
            d |= {"m_scale": self.m_scale, "v_scale": self.v_scale}
        return d

    def state_of(self, i: int) -> tuple:
        """(m, v) of tensor i in float32, in its memory order and shape [numel]."""
        at, size = self._t.query(_STATE_OFFSET + i), self.params[i].numel()
        end = at + -(-size // STATE_BLOCK) * STATE_BLOCK
        if self.state_bits == 32:
            return self.m[at:at + size], self.v[at:at + size]
        return tuple((t[at:end].float().view(-1, STATE_BLOCK) * s[at // STATE_BLOCK:end // STATE_BLOCK, None]).view(-1)[:size]
                     for t, s in ((self.m, self.m_scale), (self.v, self.v_scale)))

    def grad_norm(self, grads: Optional[Sequence] = None, max_norm: float = math.inf,
                  out: Optional[torch.Tensor] = None, stream=None):
        """(norm, scale) of the gradients (default: the parameters' ``grad``), as ``GradNorm``."""
        return self._t.norm(self._grads(grads), max_norm, out, stream)

    def step(self, grads: Optional[Sequence] = None, grad_scale: Optional[torch.Tensor] = None,
             lr: Optional[float] = None, stream=None) -> None:
        """One step with the gradients (default: the parameters' ``grad``; None: that tensor is left
        alone), each times ``grad_scale`` (one float32 on the device) if given, at rate ``lr`` (default:
        the object's).  The bias corrections go by a tensor's own count of steps: tensors that have missed some
        take a launch of their own, one for all that have missed as many.  Calls on one object must be ordered."""
        t = self._t
        t.used((self.m, self.v, self.m_scale, self.v_scale), stream)
        _lib.check("pp_adamw_step", t.native.adamw_step(
            t.list, self._grads(grads), self._written, self.state_bits, self.m, self.v, self.m_scale, self.v_scale,
            self.lr if lr is None else lr, self.betas[0], self.betas[1], self.eps, self.steps + 1, self.seed,
            grad_scale, None if stream is None else stream.cuda_stream))
        self.steps += 1

    def _grads(self, grads) -> Sequence:
        return [p.grad for p in self.params] if grads is None else grads
