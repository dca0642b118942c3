"""Plain 64-bit implementations of the handle-free operators, written from their definitions (numpy, loops where
that is plainest)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_mx4(x):
    """The values that the 4-bit microscaled form of x (float64 [rows, cols]) along its rows stands for."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    out = np.zeros_like(x)
    for c in range(0, cols, 32):
        b = x[:, c:c + 32]
        most = np.abs(b).max(1)
        fine = np.isfinite(most)
        exponent = np.full(rows, -127)
        some = fine & (most > 0)
        exponent[some] = np.maximum(np.frexp(most[some])[1] - 1 - 2, -127)
        scale = np.ldexp(1.0, exponent)[:, None]
        with np.errstate(invalid="ignore"):
            size = np.abs(b) / scale
            gap = np.abs(size[:, :, None] - GRID)
        gap = np.where(np.isnan(gap), np.inf, gap)
        best = gap.min(2, keepdims=True)
        near = gap == best                               # one element, or two at a tie: the even code wins
        code = np.where(near[:, :, 0::2].any(2), 2 * near[:, :, 0::2].argmax(2), 2 * near[:, :, 1::2].argmax(2) + 1)
        v = np.copysign(GRID[code] * scale, b)
        v[~fine] = np.nan
        out[:, c:c + 32] = v
    return out


def distill(z, index, teacher, labels=None, weight=None, lse=None, temperature=1.0, soft_weight=1.0, hard_weight=0.0):
    """(loss [rows], grad [rows, vocab]) of include/zoa.h's zoa_distill_topk in float64, row by row."""
    z = np.asarray(z, np.float64)
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    T = float(temperature)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        if w == 0.0:
            continue
        x = z[r]
        if np.isnan(x).any() or (x == np.inf).any():
            loss[r], grad[r] = np.nan, np.nan
            continue
        if (x == -np.inf).all():
            continue
        m = x.max()
        lq = (x - m) / T - np.log(np.exp((x - m) / T).sum())
        lq1 = x - m - np.log(np.exp(x - m).sum())
        q, q1 = np.exp(lq), np.exp(lq1)
        keep = [(int(i), float(t)) for i, t in zip(index[r], teacher[r]) if 0 <= i < vocab]
        if lse is None and all(t == -np.inf for _, t in keep):
            keep = []
        if keep:
            t = np.array([v for _, v in keep]) / T
            at = np.array([i for i, _ in keep])
            norm = float(lse[r]) if lse is not None else t.max() + np.log(np.exp(t - t.max()).sum())
            p = np.exp(t - norm)
            soft = sum(pk * (tk - norm - lq[i]) for pk, tk, i in zip(p, t, at) if pk > 0)
            p_rest = max(0.0, 1.0 - p.sum()) if lse is not None else 0.0
            d = q * (p.sum() + p_rest)
            np.subtract.at(d, at, p)
            if lse is not None:
                out = np.ones(vocab, bool)
                out[at] = False
                q_rest = q[out].sum()
                if p_rest > 0 and q_rest > 1e-30:
                    soft += p_rest * (np.log(p_rest) - np.log(q_rest))
                    d[out] -= p_rest * q[out] / q_rest
                else:                    # a term that is left out has no derivative
                    d -= p_rest * q
            loss[r] += soft_weight * T * T * soft
            grad[r] += soft_weight * T * d
        if labels is not None and 0 <= labels[r] < vocab:
            loss[r] -= hard_weight * lq1[labels[r]]
            grad[r] += hard_weight * q1
            grad[r, labels[r]] -= hard_weight
        loss[r] *= w
        grad[r] *= w
    return loss, grad
