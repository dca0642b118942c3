"""The operators under autograd: what it must notice (second derivatives, inputs or results changed in place)."""
import pytest
import torch

from paper_2202_06009_b200 import (DistillTopkFunction, Mx4LinearFunction, distill_topk, distill_topk_backward, distill_topk_grad, mx4_linear,
                                   mx4_matmul, mx4_quantize)
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


def test_results_written_over_saved_tensors_are_noticed():
    """`out` counts as a change in place: a node that kept the tensor refuses its backward pass."""
    p = problem(6, 64, 6, torch.float32, 2)
    x = torch.randn(6, 64, device="cuda")
    q = mx4_quantize(x)
    square = mx4_quantize(torch.randn(64, 64, device="cuda"))
    stats = distill_topk(**p, stats=True)[1]

    def writes(h):
        z = dict(p, logits=h)
        yield lambda: distill_topk_grad(**z, out=h)
        yield lambda: distill_topk_backward(torch.ones(6, device="cuda"), stats, **p, out=h)
        yield lambda: q.dequantize(torch.float32, out=h)
        yield lambda: mx4_matmul(q, square, torch.float32, out=h)
        yield lambda: mx4_linear(x, square, out=h)

    for i in range(5):
        a = torch.randn(6, 64, device="cuda").requires_grad_()
        kept = torch.exp(a)                  # its backward pass needs its result
        list(writes(kept.detach()))[i]()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.sum().backward()
    with torch.inference_mode():
        assert distill_topk_grad(**p, out=torch.empty(6, 64, device="cuda"))[1].shape == (6, 64)
        assert mx4_linear(x, square, out=torch.empty(6, 64, device="cuda")).shape == (6, 64)
