#!/usr/bin/env python
"""A student whose linear layers run in 4 bits, distilled from a stored teacher's top logits and trained by 0/1 Adam.

    python examples/distill_4bit_student.py [--steps 60] [--workers 4] [--vocab 2003] [--hidden 256] [--layers 2]

One step, for every data-parallel worker: the student's forward pass on 4-bit linear layers (Mx4LinearFunction), the loss
and the logits' gradient in one pass (distill_topk_grad), the backward pass through the same layers, and the flat
gradient, in bfloat16, into the worker's row of zoa_step_auto, which exchanges 1-bit updates on its sync steps.  The
teacher is a random table that maps a token to a distribution over the next one; what is stored of it is its best
`top` logits and its log-sum-exp.  At the end the student's weights are rounded once more and one token at a time is
generated through mx4_linear.
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2202_06009_b200 import Mx4LinearFunction, Zoa, distill_topk_grad, mx4_linear, mx4_quantize, ops_check_device  # noqa: E402


class Student:
    """Embedding, residual feed-forward layers, output projection; its parameters are views of one flat vector."""

    def __init__(self, vocab, hidden, layers):
        self.shapes = [(vocab, hidden)] + [s for _ in range(layers) for s in ((2 * hidden, hidden), (hidden, 2 * hidden))] + [(vocab, hidden)]
        self.sizes = [a * b for a, b in self.shapes]
        self.n = sum(self.sizes)

    def initial(self, generator):
        parts = [torch.randn(a, b, generator=generator, device="cuda") * (1.0 if i == 0 else b ** -0.5) for i, (a, b) in enumerate(self.shapes)]
        return torch.cat([p.flatten() for p in parts])

    def split(self, flat):
        return [p.view(s) for p, s in zip(flat[:self.n].split(self.sizes), self.shapes)]

    @staticmethod
    def forward(params, tokens):
        embedding, *layers, head = params
        h = embedding[tokens].to(torch.bfloat16)
        for up, down in zip(layers[0::2], layers[1::2]):
            h = h + Mx4LinearFunction.apply(torch.relu(Mx4LinearFunction.apply(h, up)), down)
        return Mx4LinearFunction.apply(h, head)

    @staticmethod
    def generate(params, token, count):
        """Greedy, one token at a time, on weights rounded once."""
        embedding, *layers, head = params
        layers, head = [mx4_quantize(w) for w in layers], mx4_quantize(head)
        out = []
        for _ in range(count):
            h = embedding[token].to(torch.bfloat16)
            for up, down in zip(layers[0::2], layers[1::2]):
                h = h + mx4_linear(torch.relu(mx4_linear(h, up)), down)
            token = mx4_linear(h, head).argmax(1)
            out.append(int(token))
        return out


def train(steps=60, workers=4, vocab=2003, hidden=256, layers=2, tokens=512, top=32, temperature=2.0, lr=2e-3, seed=0):
    """Returns the mean loss of every step and the tokens generated at the end."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    student = Student(vocab, hidden, layers)
    teacher = 3.0 * torch.randn(vocab, vocab, generator=g, device="cuda")            # logits of the next token
    best = teacher.topk(top, dim=1)
    index, logits = best.indices.to(torch.int32), best.values.to(torch.bfloat16)
    lse = torch.logsumexp(teacher / temperature, 1)
    losses = []
    with Zoa(student.n, workers, 0.9, 0.999, 1e-8, 4096) as opt:
        opt.set_params(student.initial(g))
        opt.set_policies(var_steps=range(steps), sync_boundaries=[0, steps // 2], sync_intervals=[1, 2])
        opt.set_grad_dtype(torch.bfloat16)
        for t in range(steps):
            grads, mean = [], 0.0
            for w in range(workers):
                params = [p.detach().requires_grad_() for p in student.split(opt.device_view("x", w))]
                batch = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
                out = student.forward(params, batch)
                label = torch.multinomial(torch.softmax(teacher[batch], 1), 1, generator=g)[:, 0].to(torch.int32)
                loss, grad = distill_topk_grad(out.detach(), index[batch], logits[batch], labels=label, teacher_lse=lse[batch],
                                               row_weight=torch.full((tokens,), 1.0 / tokens, device="cuda"), temperature=temperature,
                                               soft_weight=0.8, hard_weight=0.2)
                out.backward(grad)
                grads.append(torch.cat([p.grad.flatten() for p in params]).to(torch.bfloat16))
                mean = mean + loss.sum() / workers
            opt.step_auto(grads, lr, t)
            losses.append(mean)
        opt.check_device()
        ops_check_device()
        generated = student.generate([p.clone() for p in student.split(opt.device_view("x", 0))], torch.zeros(1, dtype=torch.long, device="cuda"), 8)
    return [float(x) for x in losses], generated


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 60), ("workers", 4), ("vocab", 2003), ("hidden", 256), ("layers", 2)):
        ap.add_argument("--" + name, type=int, default=value)
    losses, generated = train(**vars(ap.parse_args()))
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {t:4d}  loss {losses[t]:.4f}")
    print(f"step {len(losses) - 1:4d}  loss {losses[-1]:.4f}   generated {generated}")
