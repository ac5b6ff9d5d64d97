"""Weights in 4 bits with a scale per group of their rows, and products with few rows, on torch tensors: serving token by token, where
reading the weights is what takes the time.

    w = quantize(h, weights, group=128)                       # out x in, or experts x out x in; once
    y = gemm(h, x, w)                                         # x W^T: tokens x out
    ys = gemm_grouped(h, xs, w, routing.offsets)              # rows sorted by expert (experts.sort_tokens)

A value is scale * (code - zero), codes of two columns to a byte, the even one in the low half; scales (and zero points, which are 8 where there are
none) are groups x rows, in float32, bfloat16 or float16.  Matrices that were quantised elsewhere in this layout are taken as they are:
Packed(data, scale, zero, cols, group).  Everything is enqueued on the current stream of the handle's GPU, where all tensors are; checks of the C
ABI (include/ozdgemm.h) raise OzError, those made here ValueError.  Results carry no history for torch's autograd; for gradients, and for
products with many rows, unpack() gives the matrix in any float type.
"""
from __future__ import annotations

import torch

from . import ozdgemm as g
from .scaled import check_device, check_ints, check_matrix, float_type, stream_of

_FLOATS = (torch.float32, torch.bfloat16, torch.float16)


class Packed:
    """A matrix in 4 bits: data uint8 (rows x ld, or groups x rows x ld, ld a multiple of 16 with 2 ld >= cols rounded up to 32), scale and zero
    (ceil(cols / group) x rows, for each group)."""

    # desc: what the C ABI takes, addresses and strides.  What it is made of is not set to others: a matrix with another part is another Packed.
    __slots__ = ("_data", "_scale", "_zero", "_cols", "_group", "_rows", "_groups", "desc")

    def __init__(self, data, scale, zero=None, cols=None, group=128):
        cols = 2 * data.shape[-1] if cols is None else cols
        if data.dtype != torch.uint8 or scale.dtype not in _FLOATS or (zero is not None and zero.dtype != scale.dtype):
            raise ValueError("uint8 codes with float32, bfloat16 or float16 scales and zero points of their type")
        if group not in (32, 64, 128):
            raise ValueError("group: 32, 64 or 128, not %s" % (group,))
        if data.dim() not in (2, 3) or scale.dim() != data.dim() or not data.is_cuda or scale.device != data.device:
            raise ValueError("codes and scales: two or three dimensions each, on one GPU")
        rows, blocks = data.shape[-2], -(-cols // group)
        if not 0 <= cols <= 2 * data.shape[-1] or data.shape[-1] < -(-cols // 32) * 16:
            raise ValueError("rows of %d bytes do not hold %s columns, rounded up to 32" % (data.shape[-1], cols))
        if scale.shape[-2] < blocks or scale.shape[-1] < rows or scale.shape[:-2] != data.shape[:-2]:
            raise ValueError("scales %s do not cover %d x %d in groups of %d" % (tuple(scale.shape), rows, cols, group))
        if (data.shape[-1] > 1 and data.stride(-1) != 1) or (scale.shape[-1] > 1 and scale.stride(-1) != 1):
            raise ValueError("rows of codes and of scales are contiguous")
        if zero is not None and (zero.device != data.device or zero.shape != scale.shape or zero.stride() != scale.stride()):
            raise ValueError("zero points laid out as the scales")
        self._keep(data, scale, zero, cols, group)
        # a single row has no distance to the next one: what the ABI asks of it is taken
        ld = data.stride(-2) if rows > 1 else -(-data.shape[-1] // 16) * 16
        sld = scale.stride(-2) if scale.shape[-2] > 1 else max(scale.shape[-1], 1)
        batched = data.dim() == 3
        self.desc = g.oz_packed_t(data.data_ptr(), scale.data_ptr(), None if zero is None else zero.data_ptr(), ld, sld, data.stride(0) if batched else 0,
                                  scale.stride(0) if batched else 0, float_type(scale.dtype), group, 0)

    def _keep(self, data, scale, zero, cols, group):
        self._data, self._scale, self._zero, self._cols, self._group = data, scale, zero, cols, group
        self._rows, self._groups = data.shape[-2], data.shape[0] if data.dim() == 3 else 1

    data = property(lambda self: self._data)
    scale = property(lambda self: self._scale)
    zero = property(lambda self: self._zero)
    cols = property(lambda self: self._cols)
    group = property(lambda self: self._group)
    rows = property(lambda self: self._rows)
    groups = property(lambda self: self._groups)


def empty(rows, cols, group=128, zeros=False, scale_dtype=torch.float16, groups=None, device="cuda") -> Packed:
    """An uninitialised matrix in the layout that the calls here want."""
    if group not in (32, 64, 128):
        raise ValueError("group: 32, 64 or 128, not %s" % (group,))
    ld, blocks, lead = max(-(-cols // 32) * 16, 16), -(-cols // group), () if groups is None else (groups,)
    w = Packed.__new__(Packed)              # sizes and types are right by construction
    data = torch.empty(lead + (rows, ld), dtype=torch.uint8, device=device)
    scale = data.new_empty(lead + (blocks, rows), dtype=scale_dtype)
    zero = data.new_empty(lead + (blocks, rows), dtype=scale_dtype) if zeros else None
    w._keep(data, scale, zero, cols, group)
    w.desc = g.oz_packed_t(data.data_ptr(), scale.data_ptr(), zero.data_ptr() if zeros else None, ld, max(rows, 1), 0 if groups is None else rows * ld,
                           0 if groups is None else blocks * rows, float_type(scale_dtype), group, 0)
    return w


def _matrices(x, what):
    """rows, cols, ld, batch (None: a matrix) and the distance of one matrix to the next."""
    if x.dim() == 3:
        ld = check_matrix(x[0], what) if x.shape[0] else max(x.shape[2], 1)
        return x.shape[1], x.shape[2], ld, x.shape[0], x.stride(0)
    return (*x.shape, check_matrix(x, what), None, 0) if x.dim() == 2 else check_matrix(x, what)


def quantize(h: g.Handle, x, group=128, zeros=False, scale_dtype=torch.float16) -> Packed:
    """x (matrix, or groups x rows x cols) in 4 bits; zeros: with a zero point for each group, between its least and its largest value."""
    rows, cols, ld, batch, stride = _matrices(x, "x")
    kind = float_type(x.dtype)
    check_device(h, x)
    w = empty(rows, cols, group, zeros, scale_dtype, batch, x.device)
    h.call("oz_pack4", stream_of(x), rows, cols, x.data_ptr(), ld, kind, 1 if batch is None else batch, stride, w.desc)
    return w


def unpack(h: g.Handle, w: Packed, dtype=torch.float32, out=None):
    """The values of w in `dtype` (or out's)."""
    shape = w.data.shape[:-1] + (w.cols,)
    y = w.scale.new_empty(shape, dtype=dtype) if out is None else out
    rows, cols, ld, batch, stride = _matrices(y, "out")
    if y.shape != shape:
        raise ValueError("out: %s, not %s" % (tuple(shape), tuple(y.shape)))
    kind = float_type(y.dtype)
    check_device(h, w.data, w.scale, y)
    h.call("oz_unpack4", stream_of(w.data), rows, cols, y.data_ptr(), ld, kind, 1 if batch is None else batch, stride, w.desc)
    return y


def _product(h, x, w, groups, offsets, dtype, out):
    ldx = check_matrix(x, "x")
    check_device(h, x, w._data, w._scale, w._zero, offsets, out)
    (m, k), n = x.shape, w._rows
    if k != w._cols or w._groups != max(groups, 1):
        raise ValueError("x %s and %d matrices of %d x %d do not multiply" % (tuple(x.shape), w.groups, w.rows, w.cols))
    kind = float_type(x.dtype)
    if out is None:
        y, ldy, y_kind = x.new_empty((m, n), dtype=dtype), max(n, 1), kind if dtype is None else float_type(dtype)
    else:
        y, ldy, y_kind = out, check_matrix(out, "out"), float_type(out.dtype)
        if tuple(y.shape) != (m, n):
            raise ValueError("out: %d x %d, not %s" % (m, n, tuple(y.shape)))
    h.call("oz_packed_gemm", stream_of(x), groups, None if offsets is None else offsets.data_ptr(), m, n, k, x.data_ptr(), ldx, kind, w.desc, y.data_ptr(),
           ldy, y_kind)
    return y


def gemm(h: g.Handle, x, w: Packed, dtype=None, out=None):
    """x W^T in `dtype` (or out's, or x's), summed in 32 bits.  Made for few rows of x: W is read once for every 16 or 32."""
    return _product(h, x, w, 0, None, dtype, out)


def gemm_grouped(h: g.Handle, x, w: Packed, offsets, dtype=None, out=None):
    """Rows offsets[g] .. offsets[g+1] of x times W_g^T, for every group; zeros behind the last."""
    return _product(h, x, w, check_ints(offsets, "offsets").numel() - 1, offsets, dtype, out)
