"""Distillation from a teacher's top logits, on the GPU: what is kept of the teacher, the loss, its gradient.

The pruned net is retrained beside the dense net that it came from.  Of that teacher's logits ``pp_top_logits`` keeps a
row's k largest, their classes, and the log-sum-exp of the others -- little enough to be stored with the training data --
and ``distill_loss`` trains the student on them and on the labels.  ``pp_distill`` and ``pp_distill_backward`` mirror the C
entry points (include/patconv.h).  Logits are [rows, classes], float32, float16 or bfloat16, with adjacent classes; rows
may be those of a wider tensor.  Every step runs in the library's kernels; a tensor that is elsewhere or in another order
is rejected rather than copied.

    top = pp_top_logits(teacher_logits, 32, temperature=2.0)
    loss = distill_loss(student_logits, top, labels, temperature=2.0, alpha=0.7).mean()
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import _lib
from .norm import _done

MOST_KEPT, MOST_CLASSES = 256, 1 << 20


class TopLogits(NamedTuple):
    """What is kept of a teacher's rows: ``values`` [rows, k] in order, ``indices`` int32 [rows, k], and ``rest`` float32
    [rows], the log-sum-exp of the other logits over the temperature (None: the others are left out of the loss).  ``rest`` is at the
    temperature that ``pp_top_logits`` was called with, which is not held here: a loss at another one is silently another loss.
    Whoever stores top logits stores their temperature too."""
    values: torch.Tensor
    indices: torch.Tensor
    rest: Optional[torch.Tensor]


def _handle(stream):
    return None if stream is None else stream.cuda_stream


def pp_top_logits(logits: torch.Tensor, k: int, temperature: float = 1.0, stream=None) -> TopLogits:
    """The k largest logits of each row, equal ones by their classes, and the others' log-sum-exp at ``temperature``, which
    is the loss's."""
    return TopLogits(*_done("pp_top_logits", _lib.binding().top_logits(logits, k, temperature, _handle(stream))))


def pp_distill(logits: torch.Tensor, values: torch.Tensor, indices: torch.Tensor, rest: Optional[torch.Tensor] = None,
               labels: Optional[torch.Tensor] = None, temperature: float = 1.0, alpha: float = 0.5, stream=None):
    """(loss, stats) of each row: (1 - alpha) * cross entropy with the label + alpha * temperature^2 * KL divergence of the
    student's probabilities from the teacher's; stats are the float32 [rows, 5] that the backward pass needs.

    ``rest``     None: the teacher's probabilities are of the kept classes alone; else the others are one more class;
    ``labels``   int64 [rows], one outside the classes (-100) leaves a row to the teacher; None: no label's part.
    An index outside the classes (-1) is an empty place; a row with neither labels nor kept logits has loss 0, whatever its logits are.  With
    alpha 0 the teacher, with 1 the label takes no part, whatever it holds."""
    return _done("pp_distill", _lib.binding().distill(logits, values, indices, rest, labels, temperature, alpha, _handle(stream)))


def pp_distill_backward(dloss: torch.Tensor, logits: torch.Tensor, stats: torch.Tensor, values: torch.Tensor,
                        indices: torch.Tensor, rest: Optional[torch.Tensor] = None, labels: Optional[torch.Tensor] = None,
                        temperature: float = 1.0, alpha: float = 0.5, out: Optional[torch.Tensor] = None, stream=None):
    """The logits' gradient from the losses' (float32 [rows]; rows of 0 get zeros); ``out`` may be the logits themselves."""
    return _done("pp_distill_backward", _lib.binding().distill_backward(
        dloss, logits, stats, values, indices, rest, labels, temperature, alpha, out, _handle(stream)))


def distill_loss(logits: torch.Tensor, top: TopLogits, labels: Optional[torch.Tensor] = None, temperature: float = 1.0,
                 alpha: float = 0.5) -> torch.Tensor:
    """Losses of the rows, float32 [rows], as one operation that is differentiable by the logits (once), on the current stream.
    The operation is native on both sides (csrc/binding.cpp).  Captured into a graph, its leaves are such that no living eager
    graph was built from."""
    return _done("pp_distill", _lib.binding().distill_loss(logits, top.values, top.indices, top.rest, labels, temperature, alpha))
