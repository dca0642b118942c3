"""Distillation from a teacher's top logits on the GPU against the plain 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2202_06009_b200 import (DistillTopkFunction, ZoaError, binding as B, distill_topk, distill_topk_backward,
                                   distill_topk_grad)
from plain_ops import distill

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}


def problem(rows, vocab, top, dtype, seed, pad=0, offset=0, tail=False, labels=False, T=1.0):
    rng = np.random.default_rng(seed)
    wide = torch.full((rows * (vocab + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    z = wide[offset:].view(rows, vocab + pad)[:, :vocab]
    z.copy_(torch.from_numpy(rng.standard_normal((rows, vocab)) * 2))
    index = np.stack([rng.permutation(vocab)[:top] if top <= vocab else np.r_[rng.permutation(vocab), -np.ones(top - vocab)]
                      for _ in range(rows)]).astype(np.int32)
    for r in range(0, rows, 4):
        index[r, rng.integers(0, top + 1):] = -1
    teacher = torch.from_numpy(8 - np.cumsum(rng.exponential(0.5, (rows, top)), 1)).to(dtype).cuda()
    p = dict(logits=z, index=torch.from_numpy(index).cuda(), teacher=teacher, temperature=T, soft_weight=0.7,
             hard_weight=0.3 if labels else 0.0, row_weight=None, labels=None, teacher_lse=None)
    p["row_weight"] = torch.from_numpy(rng.choice([0.0, 1.0, 0.25, 3.0], rows).astype(np.float32)).cuda()
    if tail:
        known = np.where(index >= 0, as64(teacher) / T, -np.inf).max(1, initial=-30)
        p["teacher_lse"] = torch.from_numpy((known + rng.uniform(0.6, 2.0, rows)).astype(np.float32)).cuda()
    if labels:
        lab = rng.integers(0, vocab, rows).astype(np.int32)
        lab[::5] = -100
        lab[1::5] = np.where(index[1::5, 0] >= 0, index[1::5, 0], 0)      # a listed token
        lab[2::5] = vocab                                                 # outside
        p["labels"] = torch.from_numpy(lab).cuda()
    return p


def as64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def reference(p):
    return distill(as64(p["logits"]), p["index"].cpu().numpy(), as64(p["teacher"]), None if p["labels"] is None else p["labels"].cpu().numpy(),
                   as64(p["row_weight"]), as64(p["teacher_lse"]), p["temperature"], p["soft_weight"], p["hard_weight"])


def check(p, loss=None, grad=None, scale=None):
    """Tolerances.  An exponential: 2 units of its approximation (2^-22) and its argument's rounding, |argument| 2^-23
    with |argument| <= 64 here; a sum over a thread's share and 10 joins: below 200 roundings of 2^-24.  Together below
    4e-5 relative for a probability, and as much absolute for a logarithm.  Probabilities are at most 1; a tail is
    scaled by 1 / q_r, and its sum is as exact as the others."""
    want_loss, want_grad = reference(p)
    w = np.abs(as64(p["row_weight"])) if p["row_weight"] is not None else np.ones(len(want_loss))
    T, ws, wh = p["temperature"], abs(p["soft_weight"]), abs(p["hard_weight"])
    eps = 4e-5
    if loss is not None:
        got = as64(loss)
        nan = np.isnan(want_loss)
        assert np.array_equal(np.isnan(got), nan)
        inf = np.isinf(want_loss)
        assert np.array_equal(got[inf], want_loss[inf])
        ok = ~nan & ~inf
        z = as64(p["logits"])
        high = np.where(np.isfinite(z), np.abs(z), 0).max(1)
        bound = w * (ws * T * T * eps * (2 + 2 * high / T) + wh * eps * (2 + 2 * high))
        assert (np.abs(got - want_loss)[ok] <= bound[ok] + 1e-7).all(), np.max((np.abs(got - want_loss) / (bound + 1e-7))[ok])
    if grad is not None:
        if scale is not None:
            want_grad = want_grad * scale[:, None]
            w = w * np.abs(scale)
        got = as64(grad)
        nan = np.isnan(want_grad)
        assert np.array_equal(np.isnan(got), nan)
        # each of the parts of an element carries eps of itself; the parts are below |element| + 2 (q + p) each
        z = np.where(np.isfinite(as64(p["logits"])), as64(p["logits"]), -1e30)
        q = np.exp((z - z.max(1, keepdims=True)) / T)
        q /= q.sum(1, keepdims=True)
        q1 = np.exp(z - z.max(1, keepdims=True))
        q1 /= q1.sum(1, keepdims=True)
        parts = np.abs(want_grad) + w[:, None] * (2 * ws * T * q + 2 * wh * q1)
        bound = eps * parts + HALF_ULP[grad.dtype] * np.abs(want_grad) + LEAST[grad.dtype] + 1e-9 * w[:, None]
        err = np.abs(got - want_grad)
        assert (err <= bound)[~nan].all(), np.max((err / bound)[~nan])


SHAPES = [(1, 1, 1), (3, 2, 2), (4, 7, 3), (5, 33, 40), (9, 100, 8), (6, 513, 64), (7, 1000, 1), (4, 4099, 130), (3, 30522, 32),
          (2, 50257, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail,labels,T", [(False, False, 1.0), (True, False, 2.0), (False, True, 4.0), (True, True, 1.5), (True, True, 3.0)])
@pytest.mark.parametrize("rows,vocab,top", SHAPES)
def test_loss_and_gradient(rows, vocab, top, tail, labels, T, dtype):
    p = problem(rows, vocab, top, dtype, rows * vocab + top, tail=tail, labels=labels, T=T)
    loss = distill_topk(**p)
    check(p, loss)
    both, grad = distill_topk_grad(**p)
    check(p, both, grad)
    again, grad2 = distill_topk_grad(**p)
    assert torch.equal(both, again) and torch.equal(grad, grad2)
    loss, stats = distill_topk(**p, stats=True)
    check(p, loss)
    scale = np.random.default_rng(1).choice([0.0, 0.5, -2.0], rows)
    q = dict(p)
    back = distill_topk_backward(torch.from_numpy(scale.astype(np.float32)).cuda(), stats, **q)
    check(p, None, back, scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (5, 3), (8, 8), (7, 2)])
@pytest.mark.parametrize("vocab", [5, 129, 2050])
def test_strides_and_alignments(vocab, pad, offset, dtype):
    p = problem(8, vocab, 4, dtype, 3, pad, offset, tail=True, labels=True, T=2.0)
    check(p, *distill_topk_grad(**p))
    for gpad, goffset in ((0, 0), (3, 1), (pad, offset)):
        buf = torch.full((8 * (vocab + gpad) + goffset + 8,), 7.0, dtype=dtype, device="cuda")
        out = buf[goffset:goffset + 8 * (vocab + gpad)].view(8, vocab + gpad)[:, :vocab]
        loss, grad = distill_topk_grad(**p, out=out)
        check(p, loss, grad)
        assert (buf[:goffset] == 7).all() and (buf[goffset + 8 * (vocab + gpad):] == 7).all()
        assert gpad == 0 or (buf[goffset:goffset + 8 * (vocab + gpad)].view(8, -1)[:, vocab:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,rows", [(100, 5), (6001, 40), (30001, 3)])
def test_gradient_in_place_of_the_logits(vocab, rows, dtype):
    p = problem(rows, vocab, 16, dtype, 8, tail=True, labels=True, T=2.0)
    loss, grad = distill_topk_grad(**p)
    z = p["logits"].clone()
    q = dict(p, logits=z)
    loss2, grad2 = distill_topk_grad(**q, out=z)
    assert grad2.data_ptr() == z.data_ptr() and torch.equal(loss, loss2) and torch.equal(grad, z)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [60, 9000])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_rows_and_extreme_logits(vocab, tail, dtype):
    p = problem(16, vocab, 8, dtype, 4, tail=tail, labels=True, T=2.0)
    p["row_weight"] = torch.ones(16, device="cuda")
    z, index, teacher = p["logits"], p["index"], p["teacher"]
    z[:, vocab - 5:] = float("-inf")                    # a padded head
    z[0] = float("-inf")                                # nothing left
    z[1, 3] = float("nan")
    z[2, 3] = float("inf")
    z[3] = float("nan")
    p["row_weight"][3] = 0                              # not looked at
    z[4, : vocab // 2] = torch.finfo(dtype).min
    z[5] = torch.finfo(dtype).min
    z[6, 7:] = float("-inf")                            # one half of the list falls on masked tokens
    index[7] = -1                                       # no list
    teacher[8] = float("-inf")                          # a list that says nothing
    teacher[9, 1:] = float("-inf")
    index[10, 2] = vocab                                # outside
    index[11, 4:] = index[11, 0]                        # the same token again
    z[12] = torch.finfo(dtype).max
    z[13, :] = float("-inf")
    z[13, 2] = 1.0                                      # one token left
    p["labels"][13] = 2
    z[14, 0] = 60.0
    p["teacher_lse"] = None if not tail else p["teacher_lse"] + 0.5
    if tail:
        p["teacher_lse"][11] += 3
    check(p, *distill_topk_grad(**p))
    loss, stats = distill_topk(**p, stats=True)
    check(p, loss)
    check(p, None, distill_topk_backward(torch.ones(16, device="cuda"), stats, **p), np.ones(16))
    assert loss[0] == 0 and loss[3] == 0 and torch.isnan(loss[1]) and torch.isnan(loss[2])


@pytest.mark.parametrize("rows,vocab,top,dtype", [(2, 140000, 20, torch.bfloat16), (2, 70001, 20, torch.float32),
                                                  (1, 262145, 2048, torch.float16), (1, 1 << 20, 3, torch.bfloat16)])
def test_long_vocabularies(rows, vocab, top, dtype):
    p = problem(rows, vocab, top, dtype, 6, tail=True, labels=True, T=2.0)
    check(p, *distill_topk_grad(**p))


@pytest.mark.parametrize("vocab,rows", [(30522, 300), (50257, 500), (700, 3000)])
def test_many_rows(vocab, rows):
    p = problem(rows, vocab, 8, torch.bfloat16, 7, tail=True, labels=True, T=2.0)
    check(p, *distill_topk_grad(**p))


def test_offsets_past_32_bits():
    rows, vocab = 45000, 50257
    p = problem(8, vocab, 8, torch.bfloat16, 7, tail=True, labels=True)
    p["row_weight"] = torch.ones(8, device="cuda")
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[-8:] = p["logits"]
    fill = lambda t: torch.cat([torch.zeros((rows - 8,) + t.shape[1:], dtype=t.dtype, device="cuda"), t])  # noqa: E731
    big = dict(p, logits=z, index=fill(p["index"]), teacher=fill(p["teacher"]), row_weight=fill(p["row_weight"]),
               labels=fill(p["labels"]), teacher_lse=fill(p["teacher_lse"]))
    loss, grad = distill_topk_grad(**big, out=z)
    check(p, loss[-8:], grad[-8:])
    assert not loss[:-8].any() and not grad[:16].any() and not grad[-2000:-8].any()


def test_autograd_and_another_stream():
    p = problem(9, 500, 12, torch.float32, 2, tail=True, labels=True, T=2.0)
    options = {k: v for k, v in p.items() if k not in ("logits", "index", "teacher")}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        z = p["logits"].clone().requires_grad_()
        loss = DistillTopkFunction.apply(z, p["index"], p["teacher"], options)
        (loss * 0.5).sum().backward()
    s.synchronize()
    check(p, loss, z.grad, np.full(9, 0.5))


def test_sizes_of_zero_and_refusals():
    p = problem(4, 50, 6, torch.float32, 1, labels=True)
    empty = dict(p, logits=p["logits"][:0], index=p["index"][:0], teacher=p["teacher"][:0], row_weight=None, labels=None)
    loss, grad = distill_topk_grad(**empty)
    assert loss.shape == (0,) and grad.shape == (0, 50)
    for key, bad in (("logits", p["logits"].double()), ("logits", p["logits"].t()), ("index", p["index"].long()), ("index", p["index"][:3]),
                     ("teacher", p["teacher"].half()), ("teacher", p["teacher"][:, :5]), ("labels", p["labels"].long()),
                     ("row_weight", p["row_weight"][:2]), ("row_weight", p["row_weight"].double()), ("teacher_lse", torch.zeros(4))):
        with pytest.raises(ValueError):
            distill_topk(**dict(p, **{key: bad}))
    with pytest.raises(ValueError):
        distill_topk_grad(**p, out=torch.empty(4, 51, device="cuda"))
    with pytest.raises(ValueError):
        distill_topk_backward(torch.ones(4, device="cuda"), torch.ones(4, 3, device="cuda"), **p)
    for change in (dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=-1.0),
                   dict(soft_weight=float("inf")), dict(hard_weight=float("nan"))):
        with pytest.raises(ZoaError) as e:
            distill_topk(**dict(p, **change))
        assert e.value.status == B.ERR_ARG
    wide = dict(p, index=torch.zeros(4, 2049, dtype=torch.int32, device="cuda"), teacher=torch.zeros(4, 2049, device="cuda"))
    with pytest.raises(ZoaError):
        distill_topk(**wide)
    args = B.DistillArgs()
    for call in (lambda: B.zoa_distill_topk(args, 16, None, None, 0), lambda: B.lib.zoa_distill_topk(None, None, None, None, 0, None)):
        try:
            assert call() == B.ERR_ARG
        except ZoaError as e:
            assert e.status == B.ERR_ARG
