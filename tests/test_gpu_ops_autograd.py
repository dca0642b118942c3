"""The operators under autograd: what it must notice (second derivatives, inputs or results changed in place)."""
import pytest
import torch

from paper_2202_06009_b200 import DistillTopkFunction, Mx4LinearFunction
from test_gpu_distill import problem

pytestmark = pytest.mark.gpu


def test_a_second_derivative_is_refused():
    """Not offered, so not silently left out."""
    p = problem(5, 40, 6, torch.float32, 2)
    options = {"temperature": 2.0, "row_weight": p["row_weight"]}
    z = p["logits"].clone().requires_grad_()
    grad, = torch.autograd.grad(DistillTopkFunction.apply(z, p["index"], p["teacher"], options).sum(), z, create_graph=True)
    with pytest.raises(RuntimeError):
        ((grad * grad).sum() + z.sum()).backward()
    x, w = torch.randn(8, 64, device="cuda").requires_grad_(), torch.randn(48, 64, device="cuda").requires_grad_()
    dx, dw = torch.autograd.grad(Mx4LinearFunction.apply(x, w).sum(), (x, w), create_graph=True)
    for g, t in ((dx, x), (dw, w)):
        with pytest.raises(RuntimeError):
            ((g * g).sum() + t.sum()).backward()


@pytest.mark.parametrize("what", ["labels", "row_weight", "teacher_lse", "index", "teacher", "logits"])
def test_inputs_changed_before_the_backward_pass_are_noticed(what):
    p = problem(6, 50, 6, torch.float32, 2, tail=True, labels=True, T=2.0)
    options = {k: v for k, v in p.items() if k not in ("logits", "index", "teacher")}
    z = p["logits"].clone().requires_grad_()
    leaf = z * 1.0
    loss = DistillTopkFunction.apply(leaf, p["index"], p["teacher"], options)
    with torch.no_grad():
        (leaf if what == "logits" else p[what]).add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()
