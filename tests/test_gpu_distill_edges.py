"""Distillation where it can go wrong: rows without unlisted mass, tokens listed twice, far-off or broken teacher logits,
extreme temperatures, autograd's corners.  Tolerances are test_gpu_distill.check's."""
import numpy as np
import pytest
import torch

from paper_2202_06009_b200 import ZoaError, binding as B, distill_topk, distill_topk_backward, distill_topk_grad
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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top", [(300, 2000, 256), (3, 30522, 64), (40, 700, 512)])
def test_tokens_listed_twice_give_equal_bits(rows, vocab, top, dtype):
    """A token's share counts once, and the same entry's thread adds it in every call."""
    p = problem(rows, vocab, top, dtype, 14, tail=True, labels=True, T=1.5)
    p["row_weight"] = None
    half = top // 2
    p["index"][:, half:] = p["index"][:, :half].roll(5, 1)
    p["teacher_lse"] += 1.0
    loss, stats = distill_topk(**p, stats=True)
    check(p, loss)
    both, grad = distill_topk_grad(**p)
    check(p, both, grad)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(50):
        again, stats2 = distill_topk(**p, stats=True)
        both2, grad2 = distill_topk_grad(**p)
        wrong += (again != loss).sum() + (stats2 != stats).sum() + (both2 != both).sum() + (grad2 != grad).sum()
    assert wrong.item() == 0


@pytest.mark.parametrize("T", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("far", [-40000.0, 700.0, 50000.0])
def test_teacher_logits_far_from_zero(far, T):
    """A softmax does not depend on where its logits lie: the same tolerances as near zero."""
    p = problem(9, 300, 12, torch.float32, 13, labels=True, T=T)
    p["row_weight"] = None
    p["teacher"] += far
    check(p, *distill_topk_grad(**p))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("vocab,top", [(60, 8), (9000, 100)])
def test_nan_among_the_teachers_logits(vocab, top, tail, dtype):
    """It makes its row NaN, loss and gradient; in a skipped entry, or in a row of weight 0, it is not looked at."""
    p = problem(9, vocab, top, dtype, 12, tail=tail, labels=True, T=2.0)
    p["row_weight"] = torch.ones(9, device="cuda")
    p["teacher"][1, 0], p["teacher"][2, top - 1] = float("nan"), float("nan")
    p["teacher"][3, 1] = float("nan")
    p["index"][3, 1] = -1
    p["teacher"][5] = float("nan")
    p["row_weight"][5] = 0
    others = [0, 3, 4, 5, 6, 7, 8]
    q = {k: v[others] if isinstance(v, torch.Tensor) else v for k, v in p.items()}
    both, grad = distill_topk_grad(**p)
    loss, stats = distill_topk(**p, stats=True)
    back = distill_topk_backward(torch.ones(9, device="cuda"), stats, **p)
    for got in (both, loss, grad, back):
        assert torch.isnan(got[1:3]).all()
    check(q, both[others], grad[others])
    check(q, loss[others], back[others], np.ones(7))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail,labels,T", [(False, False, 0.5), (True, True, 0.5), (True, True, 0.1), (False, True, 0.02), (True, False, 0.1)])
@pytest.mark.parametrize("rows,vocab,top", [(5, 33, 40), (9, 1000, 8), (4, 30522, 32)])
def test_temperatures_below_one(rows, vocab, top, tail, labels, T, dtype):
    p = problem(rows, vocab, top, dtype, rows + top, tail=tail, labels=labels, T=T)
    check(p, *distill_topk_grad(**p))


def test_temperatures_whose_reciprocal_overflows_are_refused():
    p = problem(4, 50, 6, torch.float32, 1)
    for T in (1e-39, 1e-45, 2.0 ** -127):
        with pytest.raises(ZoaError) as e:
            distill_topk(**dict(p, temperature=T))
        assert e.value.status == B.ERR_ARG
    loss = distill_topk(**dict(p, temperature=1e-30))
    assert not torch.isnan(loss).any()


def test_pointers_that_are_not_aligned_are_refused():
    p = problem(4, 50, 6, torch.float32, 1, tail=True, labels=True)
    loss, stats = distill_topk(**p, stats=True)
    grad, ones = torch.empty(4, 50, device="cuda"), torch.ones(4, device="cuda")
    fields = dict(logits=p["logits"].data_ptr(), index=p["index"].data_ptr(), teacher=p["teacher"].data_ptr(), teacher_lse=p["teacher_lse"].data_ptr(),
                  labels=p["labels"].data_ptr(), row_weight=p["row_weight"].data_ptr(), rows=4, vocab=50, top=6, ld_logits=50, dtype=B.F32,
                  temperature=1.0, soft_weight=1.0, hard_weight=0.0)
    calls = []
    for name in ("logits", "index", "teacher", "teacher_lse", "labels", "row_weight"):
        args = B.DistillArgs(**dict(fields, **{name: fields[name] + 2}))
        calls.append(lambda args=args: B.zoa_distill_topk(args, loss.data_ptr(), None, None, 0))
    good = B.DistillArgs(**fields)
    calls += [lambda: B.zoa_distill_topk(good, loss.data_ptr() + 2, None, None, 0), lambda: B.zoa_distill_topk(good, None, stats.data_ptr() + 4, None, 0),
              lambda: B.zoa_distill_topk(good, None, None, grad.data_ptr() + 2, 50),
              lambda: B.zoa_distill_topk_backward(good, stats.data_ptr(), ones.data_ptr() + 1, grad.data_ptr(), 50)]
    for call in calls:
        with pytest.raises(ZoaError) as e:
            call()
        assert e.value.status == B.ERR_ARG


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,rows", [(100, 5), (6001, 40), (30001, 3), (50257, 700)])
def test_backward_in_place_of_the_logits(vocab, rows, dtype):
    p = problem(rows, vocab, 16, dtype, 8, tail=True, labels=True, T=2.0)
    stats = distill_topk(**p, stats=True)[1]
    scale = torch.linspace(-1, 2, rows, device="cuda")
    grad = distill_topk_backward(scale, stats, **p)
    z = p["logits"].clone()
    assert distill_topk_backward(scale, stats, **dict(p, logits=z), out=z) is z
    assert torch.equal(grad, z)
