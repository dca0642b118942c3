"""Distillation where it can go wrong: rows without unlisted mass, tokens listed twice, far-off or broken teacher logits,
extreme temperatures, autograd's corners.  Tolerances are test_gpu_distill.check's."""
import numpy as np
import pytest
import torch

from paper_2202_06009_b200 import distill_topk, distill_topk_backward, distill_topk_grad
from test_gpu_distill import TYPES, check, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [0.5, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("rows,vocab,top", [(3, 2, 2), (6, 7, 7), (5, 40, 3), (9, 900, 16), (4, 30522, 20)])
def test_gradient_without_unlisted_mass(rows, vocab, top, T, dtype):
    """With the teacher's log-sum-exp, and unlisted tokens masked out or not there, the loss leaves the term of the rest
    out; its gradient must too, and a row's gradient then adds up to nothing."""
    p = problem(rows, vocab, top, dtype, 17 * rows + top, tail=True, T=T)
    p["row_weight"] = None
    z, index = p["logits"], p["index"].long()
    keep = torch.zeros(rows, vocab + 1, dtype=torch.bool, device="cuda")
    keep.scatter_(1, torch.where(index < 0, vocab, index), True)
    keep = keep[:, :vocab] | ~keep[:, :vocab].any(1, keepdim=True)         # rows without a list stay as they are
    z.masked_fill_(~keep, float("-inf"))
    loss, grad = distill_topk_grad(**p)
    check(p, loss, grad)
    loss, stats = distill_topk(**p, stats=True)
    check(p, loss)
    back = distill_topk_backward(torch.full((rows,), -2.0, device="cuda"), stats, **p)
    check(p, None, back, np.full(rows, -2.0))
    if dtype == torch.float32:
        g = grad.double()         # the entries' tolerances together
        assert (g.sum(1).abs() <= 4e-5 * (g.abs().sum(1) + 2 * 0.7 * T)).all()
