"""4-bit microscaled matrices and the linear layer on them (include/zoa.h: zoa_mx4_*), on torch tensors.

Argument checks and marshalling only; the arithmetic runs in the library's kernels, on the current stream.  A call on
few tokens lasts as long as its Python: the checks are kept short, and calls go to the library without a layer between.
"""
import torch

from . import binding as B

_lib = B.lib
_TYPES = {torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16}
_current_device = torch.cuda.current_device
_raw_stream = torch._C._cuda_getCurrentRawStream      # of a device's current stream, without the Stream object around it
_TILE_ROWS, _TILE_COLS, _TILE_BYTES = 128, 256, B.zoa_mx4_size(1, 1)
_MAX_SIDE = 1 << 30
_changed = torch.autograd.graph.increment_version


def _matrix(x, what):
    """(type number, rows, cols, row distance) of a 2-D CUDA tensor whose rows are contiguous."""
    code = _TYPES.get(x.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, float16 or bfloat16, not {x.dtype}")
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError(f"{what} must be a 2-D CUDA tensor")
    rows, cols = x.shape
    ld, step = x.stride()
    if ld < cols or step != 1:
        if rows and ((step != 1 and cols > 1) or (ld < cols and rows > 1)):
            raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
        ld = max(ld, cols)
    return code, rows, cols, ld


def _check_result(out, rows, cols, dtype, device, what="out"):
    """The row distance of a tensor that a call will write into, which autograd is told of: a node that kept the tensor
    must not use what it then holds."""
    if out.shape != (rows, cols) or out.dtype != dtype or out.device != device:
        raise ValueError(f"{what} must be a {dtype} tensor of shape ({rows}, {cols}) on {device}")
    ld = _matrix(out, what)[3]
    _changed(out)
    return ld


def _call(fn, device, *args):
    """fn(*args, stream) with `device` current, on its current stream."""
    index = device.index
    if index == _current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status:
        B._check_ops(status)


def _size(rows, cols):
    """zoa_mx4_size."""
    if rows > _MAX_SIDE or cols > _MAX_SIDE:
        raise ValueError("a side of an Mx4 is at most 2^30")
    return -(-rows // _TILE_ROWS) * -(-cols // _TILE_COLS) * _TILE_BYTES


def _bytes(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device)


class Mx4:
    """The 4-bit microscaled form of a [rows, cols] matrix: E2M1 elements, an E8M0 scale per 32 neighbours of a row.

    `data` is one byte buffer in the library's layout.  Made by mx4_quantize / mx4_quantize_both."""
    __slots__ = ("data", "rows", "cols")

    def __init__(self, rows, cols, device="cuda", data=None):
        size = _size(rows, cols)
        if data is None:
            data = _bytes(size, device)
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
        data, rows, cols = self.data, self.rows, self.cols
        device = data.device
        if out is None:
            if dtype not in _TYPES:
                raise ValueError(f"dtype must be float32, float16 or bfloat16, not {dtype}")
            out, ld = torch.empty((rows, cols), dtype=dtype, device=device), cols
        else:
            ld = _check_result(out, rows, cols, dtype, device)
        _call(_lib.zoa_mx4_dequantize, device, data.data_ptr(), rows, cols, out.data_ptr(), _TYPES[dtype], ld)
        return out


def _form(out, rows, cols, device, what):
    if out is None:
        return Mx4(rows, cols, device)
    if out.shape != (rows, cols) or out.device != device:
        raise ValueError(f"{what} must be an Mx4 of shape ({rows}, {cols}) on {device}")
    _changed(out.data)
    return out


def mx4_quantize(x, out=None):
    """x [rows, cols] rounded along its rows."""
    code, rows, cols, ld = _matrix(x, "x")
    device = x.device
    out = _form(out, rows, cols, device, "out")
    _call(_lib.zoa_mx4_quantize, device, x.data_ptr(), code, rows, cols, ld, out.data.data_ptr(), None)
    return out


def mx4_quantize_both(x, out=None, out_t=None):
    """x rounded along its rows, and its transpose rounded along its rows (x's columns), from one read."""
    code, rows, cols, ld = _matrix(x, "x")
    device = x.device
    out = _form(out, rows, cols, device, "out")
    out_t = _form(out_t, cols, rows, device, "out_t")
    _call(_lib.zoa_mx4_quantize, device, x.data_ptr(), code, rows, cols, ld, out.data.data_ptr(), out_t.data.data_ptr())
    return out, out_t


def mx4_matmul(a, b, dtype=torch.bfloat16, out=None):
    """a [m, k] times b [n, k] transposed, both Mx4: [m, n] of `dtype`."""
    m, n, k, device = a.rows, b.rows, a.cols, a.data.device
    if k != b.cols:
        raise ValueError(f"a is {a.shape}, b is {b.shape}: their columns must agree")
    if b.data.device != device:
        raise ValueError("a and b must be on the same device")
    if out is None:
        if dtype not in _TYPES:
            raise ValueError(f"dtype must be float32, float16 or bfloat16, not {dtype}")
        out, ld = torch.empty((m, n), dtype=dtype, device=device), n
    else:
        ld = _check_result(out, m, n, dtype, device)
    _call(_lib.zoa_mx4_matmul, device, a.data.data_ptr(), b.data.data_ptr(), m, n, k, out.data_ptr(), _TYPES[dtype], ld)
    return out


def mx4_linear(x, w, out=None):
    """Q(x) w^T for activations x [tokens, in] and a weight w, Mx4 [out, in]; the result has x's type."""
    code, m, k, ldx = _matrix(x, "x")
    device, n = x.device, w.rows
    if k != w.cols:
        raise ValueError(f"x is {tuple(x.shape)}, w is {w.shape}: their columns must agree")
    if w.data.device != device:
        raise ValueError("x and w must be on the same device")
    if out is None:
        out, ld = x.new_empty((m, n)), n
    else:
        ld = _check_result(out, m, n, x.dtype, device)
    size = _lib.zoa_mx4_linear_work(m, n, k)
    work = _bytes(size, device) if size else None
    _call(_lib.zoa_mx4_linear, device, x.data_ptr(), code, m, k, ldx, w.data.data_ptr(), n, out.data_ptr(), ld,
          work.data_ptr() if size else None)
    return out


class Mx4LinearSaved:
    """What mx4_linear_backward needs of a forward step: x^T and w^T rounded along their rows, in one buffer."""
    __slots__ = ("data", "m", "n", "k", "x_dtype", "w_dtype")

    def __init__(self, data, m, n, k, x_dtype, w_dtype):
        self.data, self.m, self.n, self.k, self.x_dtype, self.w_dtype = data, m, n, k, x_dtype, w_dtype


def mx4_linear_forward(x, w):
    """Training form: y = Q(x) Q(w)^T from real x [tokens, in] and w [out, in], and what mx4_linear_backward needs
    (x and w rounded along the other axis).  The result has x's type."""
    x_type, m, k, ldx = _matrix(x, "x")
    w_type, n, k2, ldw = _matrix(w, "w")
    device = x.device
    if k != k2:
        raise ValueError(f"x is {tuple(x.shape)}, w is {tuple(w.shape)}: their columns must agree")
    if w.device != device:
        raise ValueError("x and w must be on the same device")
    y = x.new_empty((m, n))
    xt = _size(k, m)
    saved = _bytes(xt + _size(k, n), device)
    work = _bytes(_size(m, k) + _size(n, k), device)
    at = saved.data_ptr()
    _call(_lib.zoa_mx4_linear_forward, device, x.data_ptr(), x_type, ldx, w.data_ptr(), w_type, ldw, m, n, k, y.data_ptr(), n, at, at + xt,
          work.data_ptr())
    return y, Mx4LinearSaved(saved, m, n, k, x.dtype, w.dtype)


def mx4_linear_backward(dy, saved, need_dx=True, need_dw=True):
    """(dx, dw) for the gradient dy [tokens, out] of mx4_linear_forward's result, the rounding's own derivative taken
    as 1: dx = Q(dy) Q(w^T)^T, dw = Q(dy^T) Q(x^T)^T, of x's and w's types; None for one that is not needed."""
    code, m, n, ld = _matrix(dy, "dy")
    k, device = saved.k, saved.data.device
    if m != saved.m or n != saved.n or dy.device != device:
        raise ValueError(f"dy is {tuple(dy.shape)} on {dy.device}, the layer's result was ({saved.m}, {saved.n}) on {device}")
    dx = torch.empty((m, k), dtype=saved.x_dtype, device=device) if need_dx else None
    dw = torch.empty((n, k), dtype=saved.w_dtype, device=device) if need_dw else None
    if need_dx or need_dw:
        work = _bytes(_size(m, n) + _size(n, m), device)
        at = saved.data.data_ptr()
        _call(_lib.zoa_mx4_linear_backward, device, dy.data_ptr(), code, ld, m, n, k, at, at + _size(k, m),
              dx.data_ptr() if need_dx else None, _TYPES[saved.x_dtype], k, dw.data_ptr() if need_dw else None,
              _TYPES[saved.w_dtype], k, work.data_ptr())
    return dx, dw


class _OnlyFirst(torch.autograd.Function):
    @staticmethod
    def forward(ctx, grad, anchor):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("a second derivative through Mx4LinearFunction or DistillTopkFunction is not offered")


def _only_first(*grads):
    """Gradients that refuse to be differentiated (under create_graph), instead of passing for constants."""
    if not torch.is_grad_enabled():
        return grads
    return tuple(g if g is None else _OnlyFirst.apply(g, torch.empty(0, requires_grad=True)) for g in grads)


class Mx4LinearFunction(torch.autograd.Function):
    """mx4_linear_forward / mx4_linear_backward under autograd: y = Mx4LinearFunction.apply(x, w)."""

    @staticmethod
    def forward(ctx, x, w):
        y, saved = mx4_linear_forward(x, w)
        ctx.save_for_backward(saved.data)
        ctx.layer = (saved.m, saved.n, saved.k, saved.x_dtype, saved.w_dtype)
        return y

    @staticmethod
    def backward(ctx, dy):
        saved = Mx4LinearSaved(ctx.saved_tensors[0], *ctx.layer)
        ld, step = dy.stride()
        if step != 1 or ld < dy.shape[1]:       # transposed, or broadcast (a sum over tokens hands back one row for all)
            dy = dy.contiguous()
        return _only_first(*mx4_linear_backward(dy, saved, *ctx.needs_input_grad))
