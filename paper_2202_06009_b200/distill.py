"""Distillation from a teacher's top logits (include/zoa.h: zoa_distill_topk), on torch tensors.

Argument checks and marshalling only; the arithmetic runs in the library's kernels, on the current stream.
"""
import struct

import torch

from . import binding as B
from .mx4 import _call, _check_result, _matrix, _only_first

_lib = B.lib
_pack = struct.Struct("@6P4Ni3f").pack          # zoa_distill_args


def _vector(t, rows, dtype, device, what):
    if t is None:
        return 0
    if t.dtype != dtype or t.shape != (rows,) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of {rows} elements on {device}")
    return t.data_ptr()


def _args(logits, index, teacher, labels, row_weight, teacher_lse, temperature, soft_weight, hard_weight):
    """(the bytes of a zoa_distill_args, rows, vocab, device)."""
    code, rows, vocab, ld = _matrix(logits, "logits")
    device, shape = logits.device, index.shape
    if len(shape) != 2 or shape[0] != rows or index.dtype != torch.int32 or index.device != device or not index.is_contiguous():
        raise ValueError(f"index must be a contiguous int32 tensor of {rows} rows on {device}")
    if teacher.shape != shape or teacher.dtype != logits.dtype or teacher.device != device or not teacher.is_contiguous():
        raise ValueError(f"teacher must be a contiguous {logits.dtype} tensor of index's shape on {device}")
    return _pack(logits.data_ptr(), index.data_ptr(), teacher.data_ptr(),
                 _vector(teacher_lse, rows, torch.float32, device, "teacher_lse"),
                 _vector(labels, rows, torch.int32, device, "labels"),
                 _vector(row_weight, rows, torch.float32, device, "row_weight"),
                 rows, vocab, shape[1], ld, code, temperature, soft_weight, hard_weight), rows, vocab, device


def _gradient(logits, out, rows, vocab, device):
    if out is None:
        return torch.empty((rows, vocab), dtype=logits.dtype, device=device), vocab
    return out, _check_result(out, rows, vocab, logits.dtype, device, "grad")


def distill_topk(logits, index, teacher, *, labels=None, row_weight=None, teacher_lse=None, temperature=1.0, soft_weight=1.0,
                 hard_weight=0.0, stats=False):
    """The loss of every row of logits [rows, vocab] (float32 [rows]) against the teacher's tokens index (int32
    [rows, top]; an entry outside [0, vocab) is skipped) and their logits (teacher, same shape, the logits' type):

        row_weight (soft_weight temperature^2 KL(teacher || student at this temperature) + hard_weight cross_entropy(labels))

    The teacher's distribution is the softmax of the listed logits; with teacher_lse (float32 [rows], the log-sum-exp of
    the teacher's logits / temperature over its whole vocabulary) it is the true one, the unlisted tokens together being
    one more outcome.  stats=True also returns what distill_topk_backward needs (float32 [rows, 4])."""
    args, rows, _, device = _args(logits, index, teacher, labels, row_weight, teacher_lse, temperature, soft_weight, hard_weight)
    loss = torch.empty(rows, dtype=torch.float32, device=device)
    kept = torch.empty((rows, 4), dtype=torch.float32, device=device) if stats else None
    _call(_lib.zoa_distill_topk, device, args, loss.data_ptr(), kept.data_ptr() if stats else None, None, 0)
    return (loss, kept) if stats else loss


def distill_topk_grad(logits, index, teacher, *, labels=None, row_weight=None, teacher_lse=None, temperature=1.0, soft_weight=1.0,
                      hard_weight=0.0, out=None):
    """(loss, grad): distill_topk and the gradient of the sum of its rows by the logits, in one pass over them.  `out`
    receives the gradient; it may be the logits, which it then replaces."""
    args, rows, vocab, device = _args(logits, index, teacher, labels, row_weight, teacher_lse, temperature, soft_weight, hard_weight)
    loss = torch.empty(rows, dtype=torch.float32, device=device)
    grad, ld = _gradient(logits, out, rows, vocab, device)
    _call(_lib.zoa_distill_topk, device, args, loss.data_ptr(), None, grad.data_ptr(), ld)
    return loss, grad


def distill_topk_backward(grad_loss, stats, logits, index, teacher, *, labels=None, row_weight=None, teacher_lse=None,
                          temperature=1.0, soft_weight=1.0, hard_weight=0.0, out=None):
    """The gradient of sum(grad_loss * distill_topk(...)) by the logits, from the same arguments and the forward call's stats."""
    args, rows, vocab, device = _args(logits, index, teacher, labels, row_weight, teacher_lse, temperature, soft_weight, hard_weight)
    grad, ld = _gradient(logits, out, rows, vocab, device)
    if stats.shape != (rows, 4) or stats.dtype != torch.float32 or stats.device != device or not stats.is_contiguous():
        raise ValueError("stats must be the second result of distill_topk(..., stats=True)")
    _call(_lib.zoa_distill_topk_backward, device, args, stats.data_ptr(), _vector(grad_loss, rows, torch.float32, device, "grad_loss"),
          grad.data_ptr(), ld)
    return grad


_TENSORS = ("labels", "row_weight", "teacher_lse")      # of distill_topk's options


class DistillTopkFunction(torch.autograd.Function):
    """distill_topk under autograd (by the logits): DistillTopkFunction.apply(logits, index, teacher, options) with
    options a dict of distill_topk's keyword arguments."""

    @staticmethod
    def forward(ctx, logits, index, teacher, options):
        loss, stats = distill_topk(logits, index, teacher, stats=True, **options)
        # tensors among the options are kept as the others are, so that changing one before the backward pass is noticed
        ctx.numbers = {name: value for name, value in options.items() if name not in _TENSORS}
        ctx.save_for_backward(stats, logits, index, teacher, *(options.get(name) for name in _TENSORS))
        return loss

    @staticmethod
    def backward(ctx, grad_loss):
        *inputs, labels, row_weight, teacher_lse = ctx.saved_tensors
        grad, = _only_first(distill_topk_backward(grad_loss.contiguous(), *inputs, labels=labels, row_weight=row_weight,
                                                  teacher_lse=teacher_lse, **ctx.numbers))
        return grad, None, None, None
