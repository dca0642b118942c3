"""The plain 64-bit operators against their definitions: worked values, and the gradient against differences."""
import numpy as np
import pytest

from plain_ops import distill, round_mx4


def test_rounding_by_hand():
    x = np.zeros((1, 64))
    x[0, :12] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, -0.3, -6.1, 0.26]      # largest in [4, 8): scale 1
    x[0, 32:35] = [0.9, 0.1, -0.45]                                                   # scale 2^-3: 7.2, 0.8, -3.6
    got = round_mx4(x)[0]
    assert got[:12].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6, -0.5, -6, 0.5]
    assert got[32:35].tolist() == [0.75, 0.125, -0.5] and not got[35:].any()


def test_rounding_again_changes_nothing():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((20, 77)) * np.exp(3 * rng.standard_normal((20, 1)))
    once = round_mx4(x)
    assert np.array_equal(round_mx4(once), once)


def test_rounding_of_extremes():
    x = np.zeros((4, 33))
    x[0, 0], x[0, 32] = np.nan, 1.0
    x[1, 3] = np.inf
    x[2, 0] = 2.0 ** -149
    x[3, 0] = 2.0 ** -127 * 0.8
    got = round_mx4(x)
    assert np.isnan(got[0, :32]).all() and got[0, 32] == 1.0 and np.isnan(got[1, :32]).all() and got[1, 32] == 0
    assert not got[2].any() and got[3, 0] == 2.0 ** -127


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("hard", [0.0, 0.4])
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_gradient_against_differences(tail, hard, T):
    rng = np.random.default_rng(5)
    rows, vocab, top = 4, 13, 5
    z = rng.standard_normal((rows, vocab))
    index = np.stack([rng.permutation(vocab)[:top] for _ in range(rows)])
    index[1, 3:] = -1
    index[2] = -1
    teacher = rng.standard_normal((rows, top)) * 2
    lse = np.log(np.exp(np.where(index >= 0, teacher, -30) / T).sum(1)) + 0.2 if tail else None
    args = dict(labels=np.array([3, -100, 0, int(index[3, 0])]), weight=np.array([1, 0.5, 2, 1.0]), lse=lse, temperature=T,
                soft_weight=0.7, hard_weight=hard)
    _, grad = distill(z, index, teacher, **args)
    h = 1e-5
    for j in range(vocab):
        up, down = z.copy(), z.copy()
        up[:, j] += h
        down[:, j] -= h
        diff = (distill(up, index, teacher, **args)[0] - distill(down, index, teacher, **args)[0]) / (2 * h)
        # central differences: an error of h^2 / 6 times a third derivative below 10, and 2^-52 * loss / h of rounding
        assert np.abs(diff - grad[:, j]).max() < 1e-9 + 2e-10


@pytest.mark.parametrize("T", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("unlisted", ["masked", "none"])
def test_gradient_against_differences_without_unlisted_mass(unlisted, T):
    """The teacher's own log-sum-exp, and no unlisted token that the student can choose: the term of the rest is left out
    of the loss, and so of its derivative."""
    rng = np.random.default_rng(6)
    rows, top = 3, 4
    vocab = 11 if unlisted == "masked" else top
    z = rng.standard_normal((rows, vocab))
    index = np.stack([rng.permutation(vocab)[:top] for _ in range(rows)])
    if unlisted == "masked":
        kept = np.take_along_axis(z, index, 1)
        z[:] = -np.inf
        np.put_along_axis(z, index, kept, 1)
    teacher = rng.standard_normal((rows, top))
    args = dict(lse=np.log(np.exp(teacher / T).sum(1)) + 0.3, temperature=T, soft_weight=0.7)
    _, grad = distill(z, index, teacher, **args)
    # central differences, as above
    h = 1e-5
    for r in range(rows):
        for j in index[r]:
            up, down = z[r:r + 1].copy(), z[r:r + 1].copy()
            up[0, j] += h
            down[0, j] -= h
            one = dict(args, lse=args["lse"][r:r + 1])
            diff = (distill(up, index[r:r + 1], teacher[r:r + 1], **one)[0] - distill(down, index[r:r + 1], teacher[r:r + 1], **one)[0]) / (2 * h)
            assert abs(diff[0] - grad[r, j]) < 1e-9 + 2e-10
    assert np.abs(grad.sum(1)).max() < 1e-12        # a distribution less a distribution of the same mass
