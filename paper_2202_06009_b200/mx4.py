"""4-bit microscaled matrices and the linear layer on them (include/zoa.h: zoa_mx4_*), on torch tensors.

Argument checks and marshalling only; the arithmetic runs in the library's kernels, on the current stream.
"""
import torch

from . import binding as B

_TYPES = {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}


def _matrix(x, what):
    """Type number and row distance of a 2-D CUDA tensor whose rows are contiguous."""
    code = _TYPES.get(x.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, float16 or bfloat16, not {x.dtype}")
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError(f"{what} must be a 2-D CUDA tensor")
    ld, step = x.stride()
    rows, cols = x.shape
    if (step != 1 and cols > 1) or (ld < cols and rows > 1):
        raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
    return code, max(ld, cols)


def _result(out, rows, cols, dtype, like, what="out"):
    if out is None:
        out = torch.empty((rows, cols), dtype=dtype, device=like)
    elif out.shape != (rows, cols) or out.dtype != dtype or out.device != like:
        raise ValueError(f"{what} must be a {dtype} tensor of shape ({rows}, {cols}) on {like}")
    return out


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


class Mx4:
    """The 4-bit microscaled form of a [rows, cols] matrix: E2M1 elements, an E8M0 scale per 32 neighbours of a row.

    `data` is one byte buffer in the library's layout.  Made by mx4_quantize / mx4_quantize_both."""
    __slots__ = ("data", "rows", "cols")

    def __init__(self, rows, cols, device="cuda", data=None):
        size = B.zoa_mx4_size(rows, cols)
        if data is None:
            data = torch.empty(size, dtype=torch.uint8, device=device)
        elif data.dtype != torch.uint8 or not data.is_cuda or not data.is_contiguous() or data.numel() != size or data.data_ptr() % 16:
            raise ValueError(f"data must be a contiguous, 16-byte aligned uint8 CUDA tensor of {size} bytes")
        self.data, self.rows, self.cols = data, rows, cols

    @property
    def shape(self):
        return (self.rows, self.cols)

    @property
    def device(self):
        return self.data.device

    def dequantize(self, dtype=torch.bfloat16, out=None):
        """The values it stands for (exact in float32 and bfloat16)."""
        out = _result(out, self.rows, self.cols, dtype, self.data.device)
        code, ld = _matrix(out, "out")
        with torch.cuda.device(self.data.device):
            B.zoa_mx4_dequantize(self.data.data_ptr(), self.rows, self.cols, out.data_ptr(), code, ld, _stream(self.data.device))
        return out


def _form(out, rows, cols, device, what):
    if out is None:
        return Mx4(rows, cols, device)
    if out.shape != (rows, cols) or out.device != device:
        raise ValueError(f"{what} must be an Mx4 of shape ({rows}, {cols}) on {device}")
    return out


def mx4_quantize(x, out=None):
    """x [rows, cols] rounded along its rows."""
    code, ld = _matrix(x, "x")
    rows, cols = x.shape
    out = _form(out, rows, cols, x.device, "out")
    with torch.cuda.device(x.device):
        B.zoa_mx4_quantize(x.data_ptr(), code, rows, cols, ld, out.data.data_ptr(), None, _stream(x.device))
    return out


def mx4_quantize_both(x, out=None, out_t=None):
    """x rounded along its rows, and its transpose rounded along its rows (x's columns), from one read."""
    code, ld = _matrix(x, "x")
    rows, cols = x.shape
    out = _form(out, rows, cols, x.device, "out")
    out_t = _form(out_t, cols, rows, x.device, "out_t")
    with torch.cuda.device(x.device):
        B.zoa_mx4_quantize(x.data_ptr(), code, rows, cols, ld, out.data.data_ptr(), out_t.data.data_ptr(), _stream(x.device))
    return out, out_t


def mx4_matmul(a, b, dtype=torch.bfloat16, out=None):
    """a [m, k] times b [n, k] transposed, both Mx4: [m, n] of `dtype`."""
    if a.cols != b.cols:
        raise ValueError(f"a is {a.shape}, b is {b.shape}: their columns must agree")
    if a.device != b.device:
        raise ValueError("a and b must be on the same device")
    out = _result(out, a.rows, b.rows, dtype, a.device)
    code, ld = _matrix(out, "out")
    with torch.cuda.device(a.device):
        B.zoa_mx4_matmul(a.data.data_ptr(), b.data.data_ptr(), a.rows, b.rows, a.cols, out.data_ptr(), code, ld, _stream(a.device))
    return out


def mx4_linear(x, w, out=None):
    """Q(x) w^T for activations x [tokens, in] and a weight w, Mx4 [out, in]; the result has x's type."""
    code, ld = _matrix(x, "x")
    m, k = x.shape
    if k != w.cols:
        raise ValueError(f"x is {tuple(x.shape)}, w is {w.shape}: their columns must agree")
    if w.device != x.device:
        raise ValueError("x and w must be on the same device")
    n = w.rows
    out = _result(out, m, n, x.dtype, x.device)
    _, ld_out = _matrix(out, "out")
    size = B.zoa_mx4_linear_work(m, n, k)
    work = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    with torch.cuda.device(x.device):
        B.zoa_mx4_linear(x.data_ptr(), code, m, k, ld, w.data.data_ptr(), n, out.data_ptr(), ld_out,
                         work.data_ptr() if size else None, _stream(x.device))
    return out


def mx4_linear_forward(x, w):
    """Training form: y = Q(x) Q(w)^T from real x [tokens, in] and w [out, in], and what mx4_linear_backward needs
    (x and w rounded along the other axis).  The result has x's type."""
    xq, xt = mx4_quantize_both(x)
    wq, wt = mx4_quantize_both(w)
    return mx4_matmul(xq, wq, x.dtype), (xt, wt, x.dtype, w.dtype)


def mx4_linear_backward(dy, saved):
    """(dx, dw) for the gradient dy [tokens, out] of mx4_linear_forward's result, the rounding's own derivative taken
    as 1: dx = Q(dy) Q(w^T)^T, dw = Q(dy^T) Q(x^T)^T, of x's and w's types."""
    xt, wt, x_dtype, w_dtype = saved
    if dy.shape != (xt.cols, wt.cols):
        raise ValueError(f"dy is {tuple(dy.shape)}, the layer's result was ({xt.cols}, {wt.cols})")
    dyq, dyt = mx4_quantize_both(dy)
    return mx4_matmul(dyq, wt, x_dtype), mx4_matmul(dyt, xt, w_dtype)


class Mx4LinearFunction(torch.autograd.Function):
    """mx4_linear_forward / mx4_linear_backward under autograd: y = Mx4LinearFunction.apply(x, w)."""

    @staticmethod
    def forward(ctx, x, w):
        y, (xt, wt, ctx.x_dtype, ctx.w_dtype) = mx4_linear_forward(x, w)
        ctx.save_for_backward(xt.data, wt.data)
        ctx.sides = (xt.shape, wt.shape)
        return y

    @staticmethod
    def backward(ctx, dy):
        xt, wt = ctx.saved_tensors
        saved = (Mx4(*ctx.sides[0], data=xt), Mx4(*ctx.sides[1], data=wt), ctx.x_dtype, ctx.w_dtype)
        return mx4_linear_backward(dy if dy.stride(-1) == 1 else dy.contiguous(), saved)
