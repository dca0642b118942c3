"""The 4-bit layer's calls in the forms and at the sizes where they can go wrong: rests of the large product's tiles, operands that
change under repeated calls, gradients that autograd makes, empty sizes, mixed types, one-sided gradients, refusals.
Tolerances are test_gpu_mx4.assert_product's."""
import numpy as np
import pytest
import torch

from paper_2202_06009_b200 import (Mx4, Mx4LinearFunction, ZoaError, binding as B, distill_topk, distill_topk_grad, mx4_linear,
                                   mx4_linear_backward, mx4_linear_forward, mx4_matmul, mx4_quantize, mx4_quantize_both,
                                   ops_check_device)
from plain_ops import round_mx4
from test_gpu_distill import problem
from test_gpu_mx4 import ULP, as64, assert_product, data

pytestmark = pytest.mark.gpu


def assert_product_on_gpu(got, a, b, dtype):
    """test_gpu_mx4.assert_product for large results, in 64 bits on the GPU; a, b: the values of the forms."""
    a, b = a.double(), b.double()
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    rel, least = ULP[dtype]
    bound = (a.shape[1] / 8 + 8) * 2.0 ** -23 * size + rel * want.abs() + least
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rest", [1, 16, 33, 64, 100, 128, 129, 161, 200, 255])
def test_large_product_with_a_rest(rest, dtype):
    """Rows and columns of the last tiles of 256 from one to all but one; each block of a pair brings its own part."""
    k = 1100 + rest
    for m, n in ((2304, 2048 + rest), (2048 + rest, 2304), (2304 + rest, 2304 + rest)):
        a, b = data(m, k, torch.bfloat16, rest, 0.5), data(n, k, torch.bfloat16, rest + 1, 0.5, 0.1)
        qa, qb = mx4_quantize(a), mx4_quantize(b)
        assert_product_on_gpu(mx4_matmul(qa, qb, dtype), qa.dequantize(torch.float32), qb.dequantize(torch.float32), dtype)


@pytest.mark.parametrize("m,n,k", [(2304, 2304, 4096), (4096, 2049, 900), (9000, 700, 300)])
def test_large_products_of_operands_that_change(m, n, k):
    """Each call's operands replace the last call's in the same buffers: a product that began before a block's copies
    had landed would find old ones."""
    sets = [(data(m, k, torch.bfloat16, 10 * i, 0.5), data(n, k, torch.bfloat16, 10 * i + 1, 0.5, 0.1)) for i in range(2)]
    qa, qb = mx4_quantize(sets[0][0]), mx4_quantize(sets[0][1])
    want = []
    for a, b in sets:
        mx4_quantize(a, out=qa)
        mx4_quantize(b, out=qb)
        want.append(mx4_matmul(qa, qb, torch.float32))
        assert_product_on_gpu(want[-1], qa.dequantize(torch.float32), qb.dequantize(torch.float32), torch.float32)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(60):
        a, b = sets[i % 2]
        mx4_quantize(a, out=qa)
        mx4_quantize(b, out=qb)
        wrong += (mx4_matmul(qa, qb, torch.float32) != want[i % 2]).sum()
    assert wrong.item() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,k,n", [(1, 64, 48), (50, 100, 70), (300, 256, 1), (3, 33, 129)])
def test_gradients_that_autograd_broadcasts(tokens, k, n, dtype):
    """Sums and means over tokens, outputs or both hand back expanded tensors, some of whose strides are 0."""
    x, w = data(tokens, k, dtype, 1, 0.5), data(n, k, dtype, 2, 0.1, 0.05)
    v, u = data(1, n, dtype, 3)[0], data(1, tokens, dtype, 4)[0]
    losses = [lambda y: (y.sum(0) * v).sum(), lambda y: (y.mean(0) * v).sum(), lambda y: (y.sum(1) * u).sum(), lambda y: y.sum(),
              lambda y: ((y + v).sum(0) * v).sum(), lambda y: y.t().sum(0).sum(), lambda y: (y.t() @ u).sum()]
    for loss in losses:
        xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
        y = Mx4LinearFunction.apply(xa, wa)
        y.retain_grad()
        loss(y).backward()
        dx, dw = mx4_linear_backward(y.grad.contiguous(), mx4_linear_forward(x, w)[1])
        assert torch.equal(xa.grad, dx) and torch.equal(wa.grad, dw)


@pytest.mark.parametrize("need_dx,need_dw", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("m,n,k", [(0, 40, 64), (5, 0, 64), (5, 40, 0), (0, 0, 64), (0, 40, 0), (5, 0, 0), (0, 0, 0)])
def test_empty_training_steps(m, n, k, need_dx, need_dw):
    """No tokens, no outputs or no inputs: results are empty or, as empty sums, zero."""
    x, w = torch.ones(m, k, device="cuda"), torch.ones(n, k, device="cuda")
    y, saved = mx4_linear_forward(x, w)
    assert y.shape == (m, n) and not y.any()
    dx, dw = mx4_linear_backward(torch.ones(m, n, device="cuda"), saved, need_dx, need_dw)
    assert (dx is not None) == need_dx and (dw is not None) == need_dw
    for got, shape in ((dx, (m, k)), (dw, (n, k))):
        assert got is None or (got.shape == shape and not got.any())
    xa, wa = x.clone().requires_grad_(need_dx), w.clone().requires_grad_(need_dw)
    if need_dx or need_dw:
        Mx4LinearFunction.apply(xa, wa).sum().backward()
        assert xa.grad is None or (xa.grad.shape == x.shape and not xa.grad.any())
        assert wa.grad is None or (wa.grad.shape == w.shape and not wa.grad.any())


@pytest.mark.parametrize("m", [0, 1, 2, 4, 5, 40])
@pytest.mark.parametrize("n,k", [(0, 64), (40, 0), (0, 0), (0, 5000)])
def test_linear_without_outputs_or_inputs(m, n, k):
    w = mx4_quantize(torch.ones(n, k, device="cuda"))
    y = mx4_linear(torch.ones(m, k, device="cuda"), w)
    assert y.shape == (m, n) and not y.any()


def test_a_kernel_that_gave_up_is_reported_by_the_next_call():
    """Without a synchronising check: every operator refuses until zoa_ops_check_device has reported it."""
    x, w = data(200, 4096, torch.bfloat16, 1), data(200, 4096, torch.bfloat16, 2)
    a, b = mx4_quantize(x), mx4_quantize(w)
    want = mx4_matmul(a, b)
    p = problem(4, 60, 6, torch.float32, 2)
    B.zoa_ops_check_device()
    try:
        B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 20)
        B.zoa_ops_set_option(B.OPT_TEST_STOP_AFTER_TILES, 2)
        mx4_matmul(a, b)
    finally:
        B.zoa_ops_set_option(B.OPT_WAIT_LIMIT_MS, 2000)
        B.zoa_ops_set_option(B.OPT_TEST_STOP_AFTER_TILES, 0)
    torch.cuda.synchronize()
    for call in (lambda: mx4_matmul(a, b), lambda: mx4_quantize(x), lambda: a.dequantize(), lambda: mx4_linear(x, b), lambda: mx4_linear(x[:1], b),
                 lambda: mx4_linear_forward(x, w), lambda: mx4_quantize_both(x), lambda: distill_topk(**p), lambda: distill_topk_grad(**p)):
        with pytest.raises(ZoaError) as e:
            call()
        assert e.value.status == B.ERR_DEVICE
    with pytest.raises(ZoaError) as e:
        ops_check_device()
    assert e.value.status == B.ERR_DEVICE
    ops_check_device()
    assert torch.equal(mx4_matmul(a, b), want)


def test_composed_calls_check_everything_first():
    """A call that is refused has enqueued nothing: neither its work area nor a result is written."""
    m, n, k = 40, 48, 64
    x, w, dy = data(m, k, torch.float32, 1), data(n, k, torch.float32, 2), data(m, n, torch.float32, 3)
    wq = mx4_quantize(w)
    room = lambda *sizes: [torch.full((s,), 7, dtype=torch.uint8, device="cuda") for s in sizes]  # noqa: E731
    size = B.zoa_mx4_size
    xt, wt, work = room(size(k, m), size(k, n), 8 * size(128, 256))
    y, dx, dw = torch.full((m, n), 7.0, device="cuda"), torch.full((m, k), 7.0, device="cuda"), torch.full((n, k), 7.0, device="cuda")
    p = {name: t.data_ptr() for name, t in (("x", x), ("w", w), ("dy", dy), ("xt", xt), ("wt", wt), ("work", work), ("y", y), ("dx", dx),
                                            ("dw", dw), ("wq", wq.data))}

    def linear(x=p["x"], dtype=0, ldx=k, b=p["wq"], out=p["y"], ld=n, work=p["work"]):
        B.zoa_mx4_linear(x, dtype, m, k, ldx, b, n, out, ld, work)

    def forward(x=p["x"], x_type=0, ldx=k, w=p["w"], w_type=0, ldw=k, y=p["y"], ldy=n, xt=p["xt"], wt=p["wt"], work=p["work"]):
        B.zoa_mx4_linear_forward(x, x_type, ldx, w, w_type, ldw, m, n, k, y, ldy, xt, wt, work)

    def backward(dy=p["dy"], dy_type=0, ld_dy=n, xt=p["xt"], wt=p["wt"], dx=p["dx"], dx_type=0, ld_dx=k, dw=p["dw"], dw_type=0, ld_dw=k,
                 work=p["work"]):
        B.zoa_mx4_linear_backward(dy, dy_type, ld_dy, m, n, k, xt, wt, dx, dx_type, ld_dx, dw, dw_type, ld_dw, work)

    def few(b=p["wq"], out=p["y"], ld=n, ldx=k, x=p["x"]):       # rounded inside the product
        B.zoa_mx4_linear(x, 0, 2, k, ldx, b, n, out, ld, None)

    bad = [(linear, dict(x=None)), (linear, dict(dtype=3)), (linear, dict(ldx=k - 1)), (linear, dict(b=None)), (linear, dict(b=p["wq"] + 8)),
           (linear, dict(out=None)), (linear, dict(ld=n - 1)), (linear, dict(out=p["y"] + 2)), (linear, dict(work=None)), (linear, dict(work=p["work"] + 8)),
           (few, dict(b=None)), (few, dict(out=None)), (few, dict(ld=n - 1)), (few, dict(ldx=k - 1)), (few, dict(x=None)),
           (forward, dict(x=None)), (forward, dict(w=None)), (forward, dict(y=None)), (forward, dict(ldy=n - 1)), (forward, dict(y=p["y"] + 2)),
           (forward, dict(xt=None)), (forward, dict(wt=None)), (forward, dict(work=None)), (forward, dict(xt=p["xt"] + 4)), (forward, dict(wt=p["wt"] + 4)),
           (forward, dict(work=p["work"] + 4)), (forward, dict(w_type=9)), (forward, dict(x_type=9)), (forward, dict(ldw=k - 1)), (forward, dict(ldx=k - 1)),
           (backward, dict(dy=None)), (backward, dict(dy_type=9)), (backward, dict(ld_dy=n - 1)), (backward, dict(xt=None)), (backward, dict(wt=None)),
           (backward, dict(xt=p["xt"] + 4)), (backward, dict(wt=p["wt"] + 4)), (backward, dict(dx_type=9)), (backward, dict(dw_type=9)),
           (backward, dict(ld_dx=k - 1)), (backward, dict(ld_dw=k - 1)), (backward, dict(dx=p["dx"] + 2)), (backward, dict(dw=p["dw"] + 2)),
           (backward, dict(dx=None, dw=None)), (backward, dict(work=None)), (backward, dict(work=p["work"] + 8)),
           (backward, dict(dx=None, ld_dw=k - 1)), (backward, dict(dw=None, ld_dx=k - 1)), (backward, dict(dw=None, wt=None)),
           (backward, dict(dx=None, xt=None)), (backward, dict(dw_type=1, dw=p["dw"] + 1)), (backward, dict(dw_type=1, ld_dw=k - 1))]
    written = []
    for call, change in bad:
        with pytest.raises(ZoaError) as e:
            call(**change)
        assert e.value.status == B.ERR_ARG, (call.__name__, change, str(e.value))
        if not all((t == 7).all() for t in (xt, wt, work, y, dx, dw)):
            written.append((call.__name__, list(change)))
            for t in (xt, wt, work, y, dx, dw):
                t.fill_(7)
    assert not written


@pytest.mark.parametrize("x_type,w_type", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16), (torch.float16, torch.float32),
                                           (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("tokens,k,n", [(1, 33, 40), (50, 100, 70), (300, 256, 513), (1029, 1001, 1333)])
def test_training_step_of_two_types(tokens, k, n, x_type, w_type):
    """Activations in 16 bits beside the optimizer's 32-bit weights, as in training, and the other way round."""
    x, w, dy = data(tokens, k, x_type, 1, 0.5), data(n, k, w_type, 2, 0.1, 0.05), data(tokens, n, x_type, 3, 0.5, 0.01)
    y, saved = mx4_linear_forward(x, w)
    dx, dw = mx4_linear_backward(dy, saved)
    assert y.dtype == dx.dtype == x_type and dw.dtype == w_type
    x64, w64, dy64 = as64(x), as64(w), as64(dy)
    assert_product(y, round_mx4(x64), round_mx4(w64), x_type)
    assert_product(dx, round_mx4(dy64), round_mx4(w64.T), x_type)
    assert_product(dw, round_mx4(dy64.T), round_mx4(x64.T), w_type)
    # a gradient of another type than the result's
    dx2, dw2 = mx4_linear_backward(dy.float(), saved)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,k,n", [(50, 100, 70), (600, 1500, 2100)])
def test_one_gradient_alone(tokens, k, n, dtype):
    x, w, dy = data(tokens, k, dtype, 1, 0.5), data(n, k, dtype, 2, 0.1, 0.05), data(tokens, n, dtype, 3, 0.5, 0.01)
    saved = mx4_linear_forward(x, w)[1]
    dx, none = mx4_linear_backward(dy, saved, need_dw=False)
    assert none is None
    none, dw = mx4_linear_backward(dy, saved, need_dx=False)
    assert none is None
    assert_product(dx, round_mx4(as64(dy)), round_mx4(as64(w).T), dtype)
    assert_product(dw, round_mx4(as64(dy).T), round_mx4(as64(x).T), dtype)
    assert mx4_linear_backward(dy, saved, need_dx=False, need_dw=False) == (None, None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 256), (129, 511), (300, 640), (257, 129)])
def test_rounding_of_the_transpose_alone(rows, cols, dtype):
    x = data(rows, cols, dtype, rows + cols, spread=2.0)
    out_t = Mx4(cols, rows)
    B.zoa_mx4_quantize(x.data_ptr(), {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}[dtype], rows, cols, cols, None,
                       out_t.data.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert np.array_equal(as64(out_t.dequantize(torch.float32)), round_mx4(as64(x).T))
