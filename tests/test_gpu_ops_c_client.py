"""The handle-free operators from plain C: tests/c_client/ops_client.c against the plain 64-bit forms."""
import os
import subprocess

import numpy as np
import pytest

from paper_2202_06009_b200 import build as zoa_build
from plain_ops import distill, round_mx4

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")


def test_plain_c_program(tmp_path):
    lib = zoa_build.build()
    exe = str(tmp_path / "ops_client")
    subprocess.check_call(["gcc", "-std=c99", "-O1", "-Wall", "-Werror", os.path.join(ROOT, "tests", "c_client", "ops_client.c"),
                           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(CUDA, "include"),
                           "-L", os.path.dirname(lib), "-lzoa", "-L", os.path.join(CUDA, "lib64"), "-lcudart",
                           "-Wl,-rpath," + os.path.dirname(lib), "-Wl,-rpath," + os.path.join(CUDA, "lib64"), "-o", exe])
    m, n, k = 37, 205, 333
    rng = np.random.default_rng(4)
    x, w = rng.standard_normal((m, k)).astype(np.float32), (rng.standard_normal((n, k)) * 0.1).astype(np.float32)
    with open(tmp_path / "in.bin", "wb") as f:
        np.array([m, n, k], np.int64).tofile(f)
        x.tofile(f)
        w.tofile(f)
    out = subprocess.run([exe, str(tmp_path / "in.bin"), str(tmp_path / "out.bin")], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stderr
    got = np.fromfile(tmp_path / "out.bin", np.float32)
    y, loss, grad = got[:m * n].reshape(m, n), got[m * n:m * n + m], got[m * n + m:].reshape(m, n)
    a, b = round_mx4(x), round_mx4(w)
    # a binary32 sum of k exact terms in steps of 64, each step's additions counted as 8, and its rounding
    assert (np.abs(y - a @ b.T) <= (k / 8 + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 2.0 ** -24 * np.abs(y)).all()
    want_loss, want_grad = distill(y, np.zeros((m, 1), np.int64), np.zeros((m, 1)))
    # logits below 64: exponentials within 4e-5 of themselves, and so their logarithms absolutely
    assert np.abs(y).max() < 64
    assert np.abs(loss - want_loss).max() < 4e-5 * (2 + 2 * np.abs(y).max()) and np.abs(grad - want_grad).max() < 2 * 4e-5
