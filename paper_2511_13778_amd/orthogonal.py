"""Weight updates made orthogonal, on torch tensors: for a matrix of gradients (or their running mean), the matrix with the same singular vectors and
all singular values near one.

    w -= lr * orthogonalize(h, momentum)                      # out x in, or experts x out x in

Newton-Schulz steps Z <- a Z + (b A + c A^2) Z, A = Z Z^T, on the matrix units: the price of a few products of the matrix with itself.  Enqueued on the
current stream of the handle's GPU; checks of the C ABI (include/ozdgemm.h) raise OzError, those made here ValueError.  The result carries no
history for torch's autograd.
"""
from __future__ import annotations

import torch

from . import ozdgemm as g
from .packed import _matrices
from .scaled import check_device, float_type, stream_of

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalize(h: g.Handle, x, steps: int = 5, coefficients=COEFFICIENTS, eps: float = 1e-7, out=None):
    """x (matrix, or batch x rows x cols; float32, bfloat16 or float16) made orthogonal, in x's type.  bfloat16 goes through products of 11-bit operands,
    the others through products of 22 bits, which take three times as long.  out may be x."""
    rows, cols, ld, batch, stride = _matrices(x, "x")
    kind = float_type(x.dtype)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    if y.shape != x.shape or y.dtype != x.dtype:
        raise ValueError("out: %s of %s" % (tuple(x.shape), x.dtype))
    _, _, ldy, _, stride_y = _matrices(y, "out")
    check_device(h, x, out)
    a, b, c = coefficients
    need = h.orthogonalize_workspace_bytes(1 if batch is None else batch, rows, cols, kind)
    ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    h.call("oz_orthogonalize", stream_of(x), 1 if batch is None else batch, rows, cols, kind, x.data_ptr(), ld, stride, y.data_ptr(), ldy, stride_y,
           steps, a, b, c, eps, ws.data_ptr() if need else None, need)
    return y
