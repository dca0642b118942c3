"""4-bit microscaled matrices on the GPU against the plain 64-bit form: rounding and reading back bit for bit, products
within the error of a binary32 sum, the linear layer's two directions, refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2202_06009_b200 import (Mx4, Mx4LinearFunction, ZoaError, binding as B, mx4_linear, mx4_linear_backward,
                                   mx4_linear_forward, mx4_matmul, mx4_quantize, mx4_quantize_both)
from plain_ops import round_mx4

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
# Half a unit in the last place, relative, and the smallest step.
ULP = {torch.float32: (2.0 ** -24, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 0.0)}


def data(rows, cols, dtype, seed, spread=1.0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(1, cols, generator=g)) * scale
    return x.to(dtype).cuda()


def as64(t):
    return t.detach().double().cpu().numpy()


def strided(x, pad, offset):
    """The same values as rows of a wider buffer that starts `offset` elements after an aligned address."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + offset + 16,), 7.0, dtype=x.dtype, device=x.device)
    view = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


SIZES = [(1, 1), (1, 32), (3, 31), (2, 33), (5, 256), (127, 257), (128, 128), (129, 511), (33, 1000), (300, 640), (257, 129)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rounding_both_ways(rows, cols, dtype):
    x = data(rows, cols, dtype, rows * 1000 + cols, spread=2.0)
    x[rows // 2] = 0
    want, want_t = round_mx4(as64(x)), round_mx4(as64(x).T)
    assert np.array_equal(as64(mx4_quantize(x).dequantize(torch.float32)), want)
    q, qt = mx4_quantize_both(x)
    for form, ref in ((q, want), (qt, want_t)):
        for out in TYPES:
            if out == torch.float16 and dtype != torch.float16:
                continue        # values outside binary16's range
            assert np.array_equal(as64(form.dequantize(out)), ref)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (24, 8)])
def test_rounding_of_strided_rows(pad, offset, dtype):
    x = data(70, 301, dtype, pad * 10 + offset)
    v = strided(x, pad, offset)
    assert np.array_equal(as64(mx4_quantize(v).dequantize(torch.float32)), round_mx4(as64(x)))
    q, qt = mx4_quantize_both(v)
    assert np.array_equal(as64(q.dequantize(torch.float32)), round_mx4(as64(x)))
    assert np.array_equal(as64(qt.dequantize(torch.float32)), round_mx4(as64(x).T))
    out = strided(torch.zeros_like(x), pad, offset)
    q.dequantize(dtype, out=out)
    assert np.array_equal(as64(out), round_mx4(as64(x)))
    assert (out._base[:offset] == 7).all() and (pad == 0 or (out._base[offset:offset + 70 * (301 + pad)].view(70, -1)[:, 301:] == 7).all())


def test_rounding_of_extreme_values():
    x = torch.zeros(8, 96)
    x[0, 3], x[1, 40], x[2, 70] = float("nan"), float("inf"), float("-inf")
    x[3] = torch.linspace(-1, 1, 96) * 1e-39                    # subnormal
    x[4] = torch.linspace(-1, 1, 96) * 3.4e38
    x[5, :12] = torch.tensor([4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, -0.3, -6.1, 0.26])
    x[6] = torch.finfo(torch.float32).min
    x[7, 0] = 2.0 ** -149
    x = x.cuda()
    want = round_mx4(as64(x))
    q, qt = mx4_quantize_both(x)
    assert np.array_equal(as64(q.dequantize(torch.float32)), want, equal_nan=True)
    assert np.array_equal(as64(mx4_quantize(x).dequantize(torch.bfloat16)), want, equal_nan=True)
    assert np.array_equal(as64(qt.dequantize(torch.float32)), round_mx4(as64(x).T), equal_nan=True)


def test_every_bfloat16_value_next_to_a_fixed_neighbour():
    """All finite bfloat16 values, each in a block with 1.0: every exponent of the scale, every tie."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = v[torch.isfinite(v.float())]
    x = torch.zeros(v.numel(), 32, dtype=torch.bfloat16)
    x[:, 0], x[:, 17] = 1.0, v
    assert np.array_equal(as64(mx4_quantize(x.cuda()).dequantize(torch.float32)), round_mx4(as64(x)))


def assert_product(got, a, b, dtype):
    """a, b: the values that the forms stand for.  Products of two elements and two scales are exact.  A binary32 sum
    of k terms, in any order, is off by at most k 2^-23 times the sum of magnitudes even if each addition truncates;
    at most 64 terms enter one step of the sum, whose own additions are counted as 8."""
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    rel, least = ULP[dtype]
    bound = (a.shape[1] / 8 + 8) * 2.0 ** -23 * size + rel * np.abs(want) + least
    err = np.abs(as64(got) - want)
    assert (err <= bound).all(), f"worst {np.max(err / np.maximum(bound, 1e-300))} of the bound"


PRODUCTS = [(1, 1, 1), (1, 7, 32), (1, 128, 1000), (2, 300, 256), (5, 129, 511), (8, 640, 257), (9, 64, 64), (16, 200, 1024),
            (31, 131, 640), (64, 512, 512), (77, 160, 1600), (128, 128, 256), (130, 257, 300), (200, 999, 2049), (257, 515, 96),
            (513, 1030, 777), (1000, 60, 3000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype):
    a, b = data(m, k, dtype, m + n, 0.5), data(n, k, dtype, n + k + 1, 0.5, 0.1)
    qa, qb = mx4_quantize(a), mx4_quantize(b)
    va, vb = round_mx4(as64(a)), round_mx4(as64(b))
    first = mx4_matmul(qa, qb, dtype)
    assert_product(first, va, vb, dtype)
    assert torch.equal(first, mx4_matmul(qa, qb, dtype))
    y = mx4_linear(a, qb)
    assert_product(y, va, vb, dtype)


@pytest.mark.parametrize("m,n,k", [(2048, 1536, 512), (1300, 2100, 1500), (4000, 512, 100), (300, 4500, 700)])
def test_product_of_many_tiles(m, n, k):
    dtype = torch.bfloat16
    a, b = data(m, k, dtype, m, 0.5), data(n, k, dtype, n + 1, 0.5, 0.1)
    va, vb = round_mx4(as64(a)), round_mx4(as64(b))
    for out in (torch.bfloat16, torch.float32):
        assert_product(mx4_matmul(mx4_quantize(a), mx4_quantize(b), out), va, vb, out)


@pytest.mark.parametrize("m,n,k", [(2304, 2304, 512), (2500, 2337, 777), (300, 9500, 100), (19000, 200, 300), (2400, 2401, 2700), (5000, 1122, 65)])
@pytest.mark.parametrize("dtype", TYPES)
def test_large_product(m, n, k, dtype):
    a, b = data(m, k, dtype, m, 0.5), data(n, k, dtype, n + 1, 0.5, 0.1)
    va, vb = mx4_quantize(a).dequantize(torch.float32), mx4_quantize(b).dequantize(torch.float32)      # tested above
    pad = 3 if n % 2 else 16
    out = strided(torch.zeros(m, n, dtype=dtype, device="cuda"), pad, 0)
    for got in (mx4_matmul(mx4_quantize(a), mx4_quantize(b), dtype), mx4_matmul(mx4_quantize(a), mx4_quantize(b), dtype, out=out)):
        # on the GPU in 64 bits, with assert_product's bound
        want, size = va.double() @ vb.double().t(), va.double().abs() @ vb.double().abs().t()
        rel, least = ULP[dtype]
        bound = (k / 8 + 8) * 2.0 ** -23 * size + rel * want.abs() + least
        assert ((got.double() - want).abs() <= bound).all()
    assert (out._base[:m * (n + pad)].view(m, n + pad)[:, n:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 3, 20, 90, 300])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 3), (8, 8)])
def test_product_into_strided_rows(m, pad, offset, dtype):
    n, k = 203, 333
    x, w = data(m, k, dtype, 1, 0.5), data(n, k, dtype, 2, 0.5)
    q = mx4_quantize(w)
    out = strided(torch.zeros(m, n, dtype=dtype, device="cuda"), pad, offset)
    for call in (lambda: mx4_matmul(mx4_quantize(x), q, dtype, out=out), lambda: mx4_linear(strided(x, pad, offset), q, out=out)):
        out.zero_()
        call()
        assert_product(out, round_mx4(as64(x)), round_mx4(as64(w)), dtype)
        base = out._base
        assert (base[:offset] == 7).all() and (base[offset + m * (n + pad):] == 7).all()
        assert pad == 0 or (base[offset:offset + m * (n + pad)].view(m, n + pad)[:, n:] == 7).all()


@pytest.mark.parametrize("m", [1, 4, 40, 200])
def test_nan_reaches_its_rows_and_columns_only(m):
    n, k = 150, 300
    x, w = data(m, k, torch.bfloat16, 3), data(n, k, torch.bfloat16, 4)
    x[m // 2, 5], w[17, 290] = float("nan"), float("inf")
    for y in (mx4_linear(x, mx4_quantize(w)), mx4_matmul(mx4_quantize(x), mx4_quantize(w))):
        bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        bad[m // 2], bad[:, 17] = True, True
        assert torch.equal(torch.isnan(y), bad)


@pytest.mark.parametrize("m", [1, 6, 60, 300])
def test_scales_far_apart(m):
    """Blocks whose scales multiply to less than the smallest binary32 and to near the largest."""
    n, k = 140, 256
    x, w = data(m, k, torch.float32, 5), data(n, k, torch.float32, 6)
    x[:, :32] *= 1e-30
    w[:, :32] *= 1e-30
    x[:, 64:96] *= 1e17
    w[:, 64:96] *= 1e17
    assert_product(mx4_linear(x, mx4_quantize(w)), round_mx4(as64(x)), round_mx4(as64(w)), torch.float32)
    assert_product(mx4_matmul(mx4_quantize(x), mx4_quantize(w), torch.float32), round_mx4(as64(x)), round_mx4(as64(w)), torch.float32)


@pytest.mark.parametrize("tokens,k,n", [(1, 33, 40), (50, 100, 70), (300, 256, 513), (129, 1000, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_training_step(tokens, k, n, dtype):
    x, w, dy = data(tokens, k, dtype, 1, 0.5), data(n, k, dtype, 2, 0.1, 0.05), data(tokens, n, dtype, 3, 0.5, 0.01)
    y, saved = mx4_linear_forward(x, w)
    dx, dw = mx4_linear_backward(dy, saved)
    x64, w64, dy64 = as64(x), as64(w), as64(dy)
    assert_product(y, round_mx4(x64), round_mx4(w64), dtype)
    assert_product(dx, round_mx4(dy64), round_mx4(w64.T), dtype)
    assert_product(dw, round_mx4(dy64.T), round_mx4(x64.T), dtype)
    assert y.dtype == dx.dtype == dw.dtype == dtype and dx.shape == x.shape and dw.shape == w.shape
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    ya = Mx4LinearFunction.apply(xa, wa)
    ya.backward(dy)
    assert torch.equal(ya, y) and torch.equal(xa.grad, dx) and torch.equal(wa.grad, dw)


@pytest.mark.parametrize("tokens,k,n,dtype", [(600, 1500, 2100, torch.bfloat16), (3000, 2000, 2500, torch.float16), (300, 5000, 260, torch.bfloat16),
                                              (2600, 257, 4900, torch.float32), (1, 700, 900, torch.float16), (1029, 1001, 1333, torch.float32)])
def test_both_gradients_at_once(tokens, k, n, dtype):
    """The two products of the backward pass share a launch; fewer tiles than pairs of SMs, more, and uneven rests."""
    x, w, dy = data(tokens, k, dtype, 1, 0.5), data(n, k, dtype, 2, 0.1, 0.05), data(tokens, n, dtype, 3, 0.5, 0.01)
    y, saved = mx4_linear_forward(x, w)
    dx, dw = mx4_linear_backward(dy, saved)
    assert_product(dx, round_mx4(as64(dy)), round_mx4(as64(w).T), dtype)
    assert_product(dw, round_mx4(as64(dy).T), round_mx4(as64(x).T), dtype)
    again = mx4_linear_backward(dy, saved)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


def test_linear_gradient_against_differences_on_the_grid():
    """With inputs on the 4-bit grid in both directions the layer is bilinear, so differences are its gradient."""
    g = torch.Generator().manual_seed(9)
    pick = lambda *s: torch.tensor([-6.0, -4, -2, -1, 1, 2, 4, 6])[torch.randint(0, 8, s, generator=g)].cuda()  # noqa: E731
    x, w, dy = pick(40, 64), pick(48, 64), pick(40, 48)
    for t in (x, w, dy):      # every block holds a 4 or a 6: its scale is 1 whatever else changes
        t[::32], t[:, ::32] = 4.0, 4.0
    y, saved = mx4_linear_forward(x, w)
    dx, dw = mx4_linear_backward(dy, saved)
    for which, r, c in (("x", 5, 7), ("x", 33, 63), ("w", 9, 1), ("w", 47, 40)):
        t, grad = (x, dx) if which == "x" else (w, dw)
        moved = t.clone()
        moved[r, c] = 2.0 if t[r, c] != 2.0 else 1.0
        ym, _ = mx4_linear_forward(moved, w) if which == "x" else mx4_linear_forward(x, moved)
        change = ((ym - y).double() * dy.double()).sum().item()
        assert change == pytest.approx(grad[r, c].item() * (moved[r, c] - t[r, c]).item(), abs=0)     # integers: exact


def test_on_another_stream():
    x, w = data(600, 512, torch.bfloat16, 1), data(512, 512, torch.bfloat16, 2)
    want = mx4_linear(x, mx4_quantize(w))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = mx4_linear(x * 1.0, mx4_quantize(w * 1.0))
    s.synchronize()
    assert torch.equal(got, want)


def test_in_a_cuda_graph():
    x, w = data(40, 512, torch.bfloat16, 1), data(512, 512, torch.bfloat16, 2)
    q = mx4_quantize(w)
    want = mx4_linear(x, q)
    for _ in range(2):
        mx4_linear(x, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mx4_linear(x, q)
    got.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_offsets_past_32_bits():
    """A matrix of more than 2^31 elements: its first and last rows."""
    rows, cols = 70001, 32 * 1024
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    ends = torch.cat([torch.arange(3), torch.arange(rows - 3, rows)])
    x[ends.cuda()] = data(6, cols, torch.bfloat16, 11)
    want = round_mx4(as64(x[ends.cuda()]))
    q, qt = mx4_quantize_both(x)
    single = mx4_quantize(x)
    assert np.array_equal(as64(single.dequantize(torch.float32)[ends.cuda()]), want)
    del single
    back = q.dequantize(torch.bfloat16)
    assert np.array_equal(as64(back[ends.cuda()]), want)
    del back
    back = qt.dequantize(torch.bfloat16)
    assert back.shape == (cols, rows)
    last = rows - rows % 32
    assert np.array_equal(as64(back[:, last:]), round_mx4(as64(x[last:]).T))


@pytest.mark.parametrize("pad", [0, 1])
def test_product_past_32_bits(pad):
    """A result of more than 2^31 elements: its last rows, aligned and not."""
    m, n, k = 70001, 32 * 1024, 64
    a, b = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda"), data(n, k, torch.bfloat16, 2, 0.1)
    a[-3:] = data(3, k, torch.bfloat16, 3)
    out = torch.empty(m, n + pad, dtype=torch.bfloat16, device="cuda")[:, :n]
    mx4_matmul(mx4_quantize(a), mx4_quantize(b), out=out)
    assert_product(out[-3:], round_mx4(as64(a[-3:])), round_mx4(as64(b)), torch.bfloat16)
    assert not out[-300:-3].any() and not out[:300].any()


@pytest.mark.parametrize("m,n,k", [(1, 6400, 1600), (1, 9, 9000), (2, 1000, 4100), (3, 77, 70), (4, 1030, 300), (1, 33000, 256), (4, 5000, 5000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_on_few_rows(m, n, k, dtype):
    x, w = data(m, k, dtype, m, 0.5), data(n, k, dtype, n + 1, 0.5, 0.1)
    q = mx4_quantize(w)
    y = mx4_linear(x, q)
    assert_product(y, round_mx4(as64(x)), round_mx4(as64(w)), dtype)
    assert torch.equal(y, mx4_linear(x, q))


def test_sizes_of_zero():
    e = torch.empty
    assert mx4_quantize(e(0, 5, device="cuda")).dequantize().shape == (0, 5)
    w = mx4_quantize(data(40, 64, torch.float32, 1))
    assert mx4_linear(e(0, 64, device="cuda"), w).shape == (0, 40)
    y = mx4_matmul(mx4_quantize(e(3, 0, device="cuda")), mx4_quantize(e(4, 0, device="cuda")), torch.float32)
    assert y.shape == (3, 4) and not y.any()
    y = mx4_linear(e(3, 0, device="cuda"), mx4_quantize(e(4, 0, device="cuda")))
    assert y.shape == (3, 4) and not y.any()


def test_refusals_of_the_wrapper():
    x = data(4, 64, torch.float32, 1)
    q = mx4_quantize(x)
    for bad in (x.double(), x.t(), x[0], x.cpu(), x.int()):
        with pytest.raises(ValueError):
            mx4_quantize(bad)
    with pytest.raises(ValueError):
        mx4_quantize(x, out=Mx4(4, 65))
    with pytest.raises(ValueError):
        mx4_matmul(q, mx4_quantize(x[:, :63]))
    with pytest.raises(ValueError):
        mx4_linear(x[:, :63], q)
    with pytest.raises(ValueError):
        mx4_matmul(q, q, torch.bfloat16, out=torch.empty(4, 4, device="cuda"))
    with pytest.raises(ValueError):
        q.dequantize(torch.float32, out=torch.empty(4, 63, device="cuda"))
    with pytest.raises(ValueError):
        Mx4(4, 64, data=torch.empty(3, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        mx4_linear_backward(x, mx4_linear_forward(x, x)[1])


def test_refusals_of_the_library():
    x = data(4, 64, torch.float32, 1)
    q = mx4_quantize(x)
    y = torch.empty(4, 4, device="cuda")
    p, d, o = x.data_ptr(), q.data.data_ptr(), y.data_ptr()
    calls = [lambda: B.zoa_mx4_quantize(p, 9, 4, 64, 64, d, None), lambda: B.zoa_mx4_quantize(p, 0, 4, 64, 63, d, None),
             lambda: B.zoa_mx4_quantize(p, 0, 4, 64, 64, None, None), lambda: B.zoa_mx4_quantize(p + 2, 0, 4, 64, 64, d, None),
             lambda: B.zoa_mx4_quantize(p, 0, 4, 64, 64, d + 4, None), lambda: B.zoa_mx4_quantize(p, 0, 1 << 31, 64, 64, d, None),
             lambda: B.zoa_mx4_dequantize(d, 4, 64, None, 0, 64), lambda: B.zoa_mx4_dequantize(d, 4, 64, p, 0, 8),
             lambda: B.zoa_mx4_matmul(d, d, 4, 4, 64, o, 3, 4), lambda: B.zoa_mx4_matmul(d, d, 4, 4, 64, o, 0, 3),
             lambda: B.zoa_mx4_matmul(None, d, 4, 4, 64, o, 0, 4), lambda: B.zoa_mx4_matmul(d, d + 8, 4, 4, 64, o, 0, 4),
             lambda: B.zoa_mx4_matmul(d, d, 4, 4, 64, None, 0, 4), lambda: B.zoa_mx4_linear(p, 0, 4, 64, 63, d, 4, o, 4, d),
             lambda: B.zoa_ops_set_option(99, 1), lambda: B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 0)]
    before = y.clone()
    for call in calls:
        with pytest.raises(ZoaError) as e:
            call()
        assert e.value.status == B.ERR_ARG and len(str(e.value)) > 20
    assert B.lib.zoa_mx4_size(0, 5) == 0 and B.lib.zoa_mx4_size(1 << 31, 5) == 0 and B.lib.zoa_mx4_size(1, 1) == 17408
    torch.cuda.synchronize()
    assert torch.equal(before, y) or torch.isnan(before).any()
    B.zoa_ops_check_device()


@pytest.mark.parametrize("m,n", [(200, 200), (1024, 1024), (30, 500), (2400, 2400)])
def test_a_wait_that_runs_out_is_reported(m, n):
    """The copies stop early, so the product's waits run out after their limit and the status says so."""
    x, w = data(m, 4096, torch.bfloat16, 1), data(n, 4096, torch.bfloat16, 2)
    a, b = mx4_quantize(x), mx4_quantize(w)
    B.zoa_ops_check_device()
    try:
        B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 20)
        B.zoa_ops_set_option(B.OPT_TEST_STOP_AFTER_TILES, 2)
        mx4_matmul(a, b)
        with pytest.raises(ZoaError) as e:
            B.zoa_ops_check_device()
        assert e.value.status == B.ERR_DEVICE
    finally:
        B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 2000)
        B.zoa_ops_set_option(B.OPT_TEST_STOP_AFTER_TILES, 0)
    B.zoa_ops_check_device()
    assert_product(mx4_matmul(a, b), round_mx4(as64(x)), round_mx4(as64(w)), torch.bfloat16)


def test_a_wait_that_runs_out_in_both_gradients_is_reported():
    x, w = data(2000, 1500, torch.bfloat16, 1, 0.5), data(1300, 1500, torch.bfloat16, 2, 0.1, 0.05)
    dy = data(2000, 1300, torch.bfloat16, 3, 0.5, 0.01)
    y, saved = mx4_linear_forward(x, w)
    want = mx4_linear_backward(dy, saved)
    B.zoa_ops_check_device()
    try:
        B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 20)
        B.zoa_ops_set_option(B.OPT_TEST_STOP_AFTER_TILES, 3)
        mx4_linear_backward(dy, saved)
        with pytest.raises(ZoaError) as e:
            B.zoa_ops_check_device()
        assert e.value.status == B.ERR_DEVICE
    finally:
        B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 2000)
        B.zoa_ops_set_option(B.OPT_TEST_STOP_AFTER_TILES, 0)
    B.zoa_ops_check_device()
    got = mx4_linear_backward(dy, saved)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_structure_sizes_match_the_header():
    assert ctypes.sizeof(B.DistillArgs) == 6 * 8 + 4 * 8 + 4 * 4
