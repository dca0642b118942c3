"""0/1 Adam optimizer step for W simulated data-parallel workers on one B200.

`binding` exposes the C ABI of include/zoa.h (libzoa.so, hand-written sm_100a
kernels); `Zoa` is a small convenience wrapper around a handle that takes
torch tensors for the gradients; `synth` builds the seeded synthetic workloads.
`mx4` (4-bit microscaled matrices and the linear layer on them) and `distill` (the loss
against a teacher's top logits) make such gradients; `ops_check_device` waits for the device and
says whether one of their kernels gave up on a bounded wait.
"""
from . import binding
from .binding import ZoaError, zoa_ops_check_device as ops_check_device
from .distill import DistillTopkFunction, distill_topk, distill_topk_backward, distill_topk_grad
from .mx4 import (Mx4, Mx4LinearFunction, mx4_linear, mx4_linear_backward, mx4_linear_forward, mx4_matmul, mx4_quantize,
                  mx4_quantize_both)
from .optimizer import Zoa

__all__ = ["binding", "Zoa", "ZoaError", "Mx4", "Mx4LinearFunction", "mx4_linear", "mx4_linear_backward", "mx4_linear_forward",
           "mx4_matmul", "mx4_quantize", "mx4_quantize_both", "DistillTopkFunction", "distill_topk", "distill_topk_backward",
           "distill_topk_grad", "ops_check_device"]
