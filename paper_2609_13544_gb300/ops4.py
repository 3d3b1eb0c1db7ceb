"""Binding of the 4-bit products and of the root-mean-square norm (include/peat_ops.h), and the layers made of them.

``peat_quantize_f4`` rounds a matrix to 4-bit floating point with a scale for each block, ``peat_matmul_f4`` multiplies
two such matrices, ``peat_product_f4`` rounds what is not 4-bit yet on the way; ``Linear4`` is the layer as a playback
step replays it, beside ``Linear8``.  ``peat_rmsnorm`` is the norm in front of such a layer, with the residual stream's
addition, whose output comes in 8 bits as ``Linear8.forward_rounded`` takes it (and as values, and not rounded);
``peat_rmsnorm_backward`` has its gradients.

Formats: "mxfp4" (blocks of 32, powers of two) and "nvfp4" (blocks of 16, 8-bit floats, and a float32 scale a row).
As in the rest of the binding a ``_raw`` function fills outputs that the caller holds, the plain ones allocate them, and
all of them only enqueue work on the stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from .ops import (LinearBase, OperandF4, _as_rows, _call, _code, _code_or_int8, _matrix, _on, _padded, _stream, _vector,
                  INT8)

F4_FORMATS = {"mxfp4": 0, "nvfp4": 1}
F4_BLOCK = {"mxfp4": 32, "nvfp4": 16}
F4 = 102


def _format(name: str) -> int:
    code = F4_FORMATS.get(name)
    if code is None:
        raise ValueError(f"unknown format {name!r}: mxfp4 or nvfp4")
    return code


def f4_scale_bytes(rows: int, blocks: int) -> int:
    """Bytes of the block scales of a matrix of `rows` rows of `blocks` blocks."""
    return -(-rows // 128) * -(-blocks // 4) * 512


_uint8 = None


def _is_bytes(t) -> bool:
    global _uint8
    if _uint8 is None:
        import torch
        _uint8 = torch.uint8
    return t.dtype is _uint8


class Float4:
    """A matrix [rows, cols] in 4 bits: q uint8 [rows, cols / 2], two codes a byte, its rows starting on 16-byte
    boundaries; block_scale uint8, in tiles (include/peat_ops.h); scale float32 [rows] (nvfp4; None: 1).  Made once and
    passed to every product; it holds the tensors."""

    __slots__ = ("format", "q", "block_scale", "scale", "rows", "cols", "device", "code", "args", "operand")

    def __init__(self, format: str, q, block_scale, scale=None):
        self.code = _format(format)
        if not q.is_cuda or q.dim() != 2 or not _is_bytes(q):
            raise ValueError("q must be a CUDA matrix of uint8")
        self.device = q.get_device()
        ld = _matrix(self, q, "q")
        self.format, self.q, self.block_scale, self.scale = format, q, block_scale, scale
        self.rows, self.cols = q.shape[0], 2 * q.shape[1]
        block = F4_BLOCK[format]
        if self.cols % block:
            raise ValueError(f"a row of q must be whole blocks, {block // 2} bytes each")
        need = f4_scale_bytes(self.rows, self.cols // block)
        if (not _is_bytes(block_scale) or not block_scale.is_contiguous() or block_scale.numel() < need
                or block_scale.get_device() != self.device):
            raise ValueError(f"block_scale must be {need} contiguous bytes (uint8) on q's device")
        if scale is not None and self.code == 0:
            raise ValueError("mxfp4 has no float32 scales")
        s = _vector(self, scale, self.rows, "scale")
        self.args = q.data_ptr(), ld, block_scale.data_ptr(), s
        self.operand = OperandF4(q.data_ptr(), block_scale.data_ptr(), s, self.rows, self.cols, ld, F4, 0)

    def values(self):
        """The float32 values that it stands for [rows, cols]."""
        import torch
        block = F4_BLOCK[self.format]
        blocks, tall = self.cols // block, -(-self.rows // 128)
        wide = -(-blocks // 4)
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=self.q.device)
        code = torch.stack([self.q & 15, self.q >> 4], 2).view(self.rows, blocks, block).long()
        v = torch.where(code > 7, -table[code & 7], table[code & 7])
        s = self.block_scale[: f4_scale_bytes(self.rows, blocks)].view(tall, wide, 32, 4, 4).permute(0, 3, 2, 1, 4)
        s = s.reshape(tall * 128, 4 * wide)[: self.rows, :blocks]
        if self.code == 0:
            bits = torch.where(s == 0, 1 << 22, torch.where(s == 255, 0x7fc00000, s.int() << 23)).int()
            return (v * bits.view(torch.float32)[:, :, None]).view(self.rows, self.cols)
        v = (v * s.contiguous().view(torch.float8_e4m3fn).float()[:, :, None]).view(self.rows, self.cols)
        return v if self.scale is None else v * self.scale[:, None]


def peat_quantize_f4_raw(h, x, format: str, axis: int = 0, q=None, block_scale=None, scale=None, values=None,
                         stream=None) -> None:
    """peat_quantize_f4 on preallocated device outputs: q uint8 [rows, bytes of whole blocks] (axis 1: of x's
    transpose), block_scale uint8, scale float32 [rows] (nvfp4), values of x's shape and type; each may be None, but
    not both of q and values."""
    code = _format(format)
    ldx = _matrix(h, x, "x")
    rows, cols = x.shape
    across, k = (cols, rows) if axis else (rows, cols)
    ldq = ldv = 0
    bs = None
    if q is not None or block_scale is not None:
        blocks = -(-k // F4_BLOCK[format])
        if q is not None:
            ldq = _matrix(h, q, "q")
            if not _is_bytes(q) or tuple(q.shape) != (across, blocks * (F4_BLOCK[format] // 2)):
                raise ValueError("q must be uint8, a row of whole blocks for each row (axis 1: column) of x")
        if block_scale is not None:
            need = f4_scale_bytes(across, blocks)
            if (not _is_bytes(block_scale) or not block_scale.is_contiguous() or block_scale.numel() < need
                    or block_scale.get_device() != h.device):
                raise ValueError(f"block_scale must be {need} contiguous bytes (uint8) on the handle's device")
            bs = block_scale.data_ptr()
    if values is not None:
        ldv = _matrix(h, values, "values")
        if values.dtype != x.dtype or values.shape != x.shape:
            raise ValueError("values must have x's shape and type")
    _call(h, "peat_quantize_f4", x.data_ptr(), rows, cols, ldx, _code(x), code, axis, None if q is None else q.data_ptr(),
          ldq, bs, _vector(h, scale, across, "scale"), None if values is None else values.data_ptr(), ldv, _stream(h, stream))


def peat_quantize_f4(h, x, format: str = "mxfp4", axis: int = 0, stream=None) -> Float4:
    """x in 4 bits, with blocks along its rows (axis 0) or down its columns (axis 1: of its transpose)."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must have two dimensions")
    _format(format)
    rows, k = x.shape if axis == 0 else (x.shape[1], x.shape[0])
    blocks = -(-k // F4_BLOCK[format])
    with _on(stream):
        q = _padded(rows, blocks * (F4_BLOCK[format] // 2), x.device).view(torch.uint8)
        block_scale = torch.empty(f4_scale_bytes(rows, blocks), dtype=torch.uint8, device=x.device)
        scale = torch.empty(rows, dtype=torch.float32, device=x.device) if format == "nvfp4" else None
        peat_quantize_f4_raw(h, x, format, axis, q, block_scale, scale, None, stream)
        return Float4(format, q, block_scale, scale)


def _same_kind(h, a: Float4, b: Float4) -> None:
    if a.code != b.code:
        raise ValueError("a and b differ in their format")
    if a.device != h.device or b.device != h.device:
        raise ValueError("a and b must be on the handle's device")


def peat_matmul_f4_raw(h, a: Float4, b: Float4, out, bias=None, stream=None) -> None:
    """peat_matmul_f4 of a [M, K] and b [N, K] into out [M, N] (float32, float16 or bfloat16)."""
    _same_kind(h, a, b)
    if a.cols != b.cols:
        raise ValueError("a and b differ in their row length")
    ldo = _matrix(h, out, "out")
    if out.shape != (a.rows, b.rows):
        raise ValueError("out must be [rows of a, rows of b]")
    _call(h, "peat_matmul_f4", a.code, *a.args, *b.args, _vector(h, bias, b.rows, "bias"), a.rows, b.rows, a.cols,
          out.data_ptr(), ldo, _code(out), _stream(h, stream))


def peat_matmul_f4(h, a: Float4, b: Float4, bias=None, out_dtype=None, stream=None):
    """sum over k of a[m, k] b[n, k] + bias[n] as out_dtype (float32 unless given)."""
    import torch
    with _on(stream):
        out = torch.empty(a.rows, b.rows, dtype=out_dtype or torch.float32, device=a.q.device)
        peat_matmul_f4_raw(h, a, b, out, bias, stream)
    return out


def _operand4(h, t, axis: int, name: str):
    """(structure, rows of the operand, its K) of a matrix that is in 4 bits or is rounded to them."""
    if isinstance(t, Float4):
        if axis != 0:
            raise ValueError(f"{name} is in 4 bits already: axis 0")
        return t.operand, t.rows, t.cols
    ld = _matrix(h, t, name)
    rows, cols = t.shape
    op = OperandF4(t.data_ptr(), None, None, rows, cols, ld, _code(t), axis)
    return (op, cols, rows) if axis else (op, rows, cols)


def _operands4(h, a, b, a_axis: int, b_axis: int, format: Optional[str]):
    """The format's code, the structures of both operands, and M and N."""
    code = None if format is None else _format(format)
    for t in (a, b):
        if isinstance(t, Float4):
            if code is not None and t.code != code:
                raise ValueError("an operand is of another format")
            if t.device != h.device:
                raise ValueError("the operands must be on the handle's device")
            code = t.code
    if code is None:
        raise ValueError("no operand is in 4 bits yet: a format is needed")
    block = 16 if code else 32
    x, M, ka = _operand4(h, a, a_axis, "a")
    y, N, kb = _operand4(h, b, b_axis, "b")
    if -(-ka // block) != -(-kb // block) or (ka != kb and not isinstance(a, Float4) and not isinstance(b, Float4)):
        raise ValueError("a and b differ in their row length")
    return code, x, y, M, N


def peat_product_f4_raw(h, a, b, out, format: Optional[str] = None, a_axis: int = 0, b_axis: int = 0, bias=None,
                        stream=None) -> None:
    """peat_product_f4 into out [M, N] (float32, float16 or bfloat16): each operand a Float4, or a float matrix that is
    rounded to `format` (None: the other operand's) along its rows (axis 0) or columns (axis 1; its transpose is the
    operand)."""
    code, x, y, M, N = _operands4(h, a, b, a_axis, b_axis, format)
    ldo = _matrix(h, out, "out")
    if out.shape[0] != M or out.shape[1] != N:
        raise ValueError("out must be [rows of a, rows of b]")
    _call(h, "peat_product_f4", code, ctypes.byref(x), ctypes.byref(y), _vector(h, bias, N, "bias"), out.data_ptr(), ldo,
          _code(out), _stream(h, stream))


def peat_product_f4(h, a, b, format: Optional[str] = None, a_axis: int = 0, b_axis: int = 0, bias=None, out_dtype=None,
                    stream=None):
    """The product as a new tensor of out_dtype (float32 unless given)."""
    if stream is not None:
        with _on(stream):
            return peat_product_f4(h, a, b, format, a_axis, b_axis, bias, out_dtype)
    import torch
    code, x, y, M, N = _operands4(h, a, b, a_axis, b_axis, format)
    out = torch.empty(M, N, dtype=out_dtype or torch.float32, device=torch.device("cuda", h.device))
    _call(h, "peat_product_f4", code, ctypes.byref(x), ctypes.byref(y), _vector(h, bias, N, "bias"), out.data_ptr(), N,
          _code(out), _stream(h, None))
    return out


class Linear4(LinearBase):
    """y = x w^T with w [out, in] held in 4 bits of `format`, with blocks along its rows for the forward product and
    down its columns for the input gradient; x and the output gradient are rounded as they come (along their rows, or,
    for the weight gradient, down their columns).  Inputs are float32, float16 or bfloat16 with any leading dimensions
    and strides; the layer keeps none of them."""

    def __init__(self, h, weight, format: str = "mxfp4", stream=None):
        self.format, self._code = format, _format(format)
        super().__init__(h, weight, stream)

    def _hold(self, weight, axis: int, stream):
        return peat_quantize_f4(self.h, weight, self.format, axis, stream)

    def _take(self, x, name: str):
        return _operand4(self.h, x, 0, name)[0]

    def _multiply(self, a, b, *rest) -> None:
        _call(self.h, "peat_product_f4", self._code, ctypes.byref(a), ctypes.byref(b.operand), *rest)

    def _columns(self, g, x):
        return peat_product_f4(self.h, g, x, self.format, 1, 1)


# ---------------------------------------------------------------------------
# root-mean-square norm
# ---------------------------------------------------------------------------
def _like(h, t, shape, dtype, name: str):
    """(pointer, row distance) of an optional matrix of x's shape and type."""
    if t is None:
        return None, shape[1]
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must have x's shape and type")
    return t.data_ptr(), shape[1] if t.is_contiguous() and t.get_device() == h.device else _matrix(h, t, name)


def _norm_weight(h, weight, cols: int, dtype):
    """(pointer, type code) of a norm's weights."""
    if weight.shape != (cols,) or not weight.is_contiguous() or weight.get_device() != h.device:
        raise ValueError(f"weight must be a contiguous vector of {cols} elements on the handle's device")
    code = _code(weight)
    if code != 0 and weight.dtype is not dtype:
        raise TypeError("weight must be of x's type or float32")
    return weight.data_ptr(), code


def peat_rmsnorm_raw(h, x, weight, eps: float = 1e-6, residual=None, sum=None, y=None, q=None, scale=None, values=None,
                     rstd=None, stream=None) -> None:
    """peat_rmsnorm of x [rows, cols] on preallocated device outputs: sum (x + residual), y and values of x's shape and
    type, q int8 of x's shape, scale and rstd float32 [rows]; each may be None, but not all.  sum may be x or residual
    itself."""
    ldx = _matrix(h, x, "x")
    shape, dtype = x.shape, x.dtype
    rows, cols = shape
    ldq, qp = cols, None
    if q is not None:
        ldq, qp = _matrix(h, q, "q"), q.data_ptr()
        if _code_or_int8(q) != INT8 or q.shape != shape:
            raise ValueError("q must be int8 of x's shape")
    _call(h, "peat_rmsnorm", x.data_ptr(), ldx, *_like(h, residual, shape, dtype, "residual"),
          *_norm_weight(h, weight, cols, dtype), rows, cols, _code(x), eps, *_like(h, sum, shape, dtype, "sum"),
          *_like(h, y, shape, dtype, "y"), qp, ldq, _vector(h, scale, rows, "scale"),
          *_like(h, values, shape, dtype, "values"), _vector(h, rstd, rows, "rstd"), _stream(h, stream))


def peat_rmsnorm(h, x, weight, eps: float = 1e-6, residual=None, rounded: bool = True, stream=None) -> dict:
    """The norm of x (+ residual) [rows, cols]: a dict of sum (x itself without a residual), rstd, and q and scale (the
    output in 8 bits), or, with rounded False, y."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must have two dimensions")
    with _on(stream):
        rows, cols = x.shape
        got = {"sum": x if residual is None else torch.empty_like(x, memory_format=torch.contiguous_format),
               "rstd": torch.empty(rows, dtype=torch.float32, device=x.device)}
        if rounded:
            got["q"] = _padded(rows, cols, x.device)
            got["scale"] = torch.empty(rows, dtype=torch.float32, device=x.device)
        else:
            got["y"] = torch.empty_like(x, memory_format=torch.contiguous_format)
        peat_rmsnorm_raw(h, x, weight, eps, residual, None if residual is None else got["sum"], got.get("y"), got.get("q"),
                         got.get("scale"), None, got["rstd"], stream)
    return got


def peat_rmsnorm_backward_raw(h, grad, x, weight, rstd, grad_x=None, grad_weight=None, grad_sum=None, stream=None) -> None:
    """peat_rmsnorm_backward from grad = dL/dy, x (the norm's sum) and rstd on preallocated outputs: grad_x of x's shape
    and type (grad or grad_sum itself, if need be), grad_weight float32 [cols]; not both None."""
    if rstd is None or grad is None:
        raise ValueError("grad and rstd are needed")
    ldx = _matrix(h, x, "x")
    shape, dtype = x.shape, x.dtype
    rows, cols = shape
    _call(h, "peat_rmsnorm_backward", *_like(h, grad, shape, dtype, "grad"), *_like(h, grad_sum, shape, dtype, "grad_sum"),
          x.data_ptr(), ldx, *_norm_weight(h, weight, cols, dtype), _vector(h, rstd, rows, "rstd"), rows, cols, _code(x),
          *_like(h, grad_x, shape, dtype, "grad_x"), _vector(h, grad_weight, cols, "grad_weight"), _stream(h, stream))


def peat_rmsnorm_backward(h, grad, x, weight, rstd, grad_sum=None, stream=None):
    """(grad_x of x's type, grad_weight float32): the gradients of the norm's input (and of its residual) and weight."""
    import torch
    with _on(stream):
        grad_x = torch.empty_like(x, memory_format=torch.contiguous_format)
        grad_weight = torch.empty(x.shape[1], dtype=torch.float32, device=x.device)
        peat_rmsnorm_backward_raw(h, grad, x, weight, rstd, grad_x, grad_weight, grad_sum, stream)
    return grad_x, grad_weight


class RMSNorm8:
    """The norm in front of a layer that is replayed in 8 bits: y = (x + residual) / sqrt(mean of squares + eps) weight,
    its output as ``Linear8.forward_rounded`` takes it.  Inputs have any leading dimensions and strides; the layer holds
    its weight [cols] and none of them."""

    def __init__(self, h, weight, eps: float = 1e-6):
        self.h, self.weight, self.eps = h, weight, eps
        self.cols = weight.shape[0]

    def _rows(self, t, name: str):
        if t.shape[-1:] != (self.cols,):
            raise ValueError(f"the last dimension of {name} must be {self.cols}")
        return _as_rows(t, self.cols)

    def forward(self, x, residual=None, stream=None) -> dict:
        """sum [..., cols] of x's type, rstd [...], q int8 [..., cols] and scale [...]."""
        if stream is not None:
            with _on(stream):
                return self.forward(x, residual)
        if residual is not None and residual.shape != x.shape:
            raise ValueError("residual must have x's shape")
        got = peat_rmsnorm(self.h, self._rows(x, "x"), self.weight, self.eps,
                           None if residual is None else self._rows(residual, "residual"))
        lead = x.shape[:-1]
        return {k: v.view(*lead, self.cols) if v.dim() == 2 else v.view(lead) for k, v in got.items()}

    def backward(self, grad, sum, rstd, grad_sum=None, stream=None):
        """(the gradient of x and residual, of x's type and shape, the weight's in float32) from grad = dL/dy and forward's
        sum and rstd."""
        if stream is not None:
            with _on(stream):
                return self.backward(grad, sum, rstd, grad_sum)
        if grad.shape != sum.shape or (grad_sum is not None and grad_sum.shape != sum.shape):
            raise ValueError("grad and grad_sum must have sum's shape")
        grad_x, grad_weight = peat_rmsnorm_backward(
            self.h, self._rows(grad, "grad"), self._rows(sum, "sum"), self.weight, rstd.reshape(-1),
            None if grad_sum is None else self._rows(grad_sum, "grad_sum"))
        return grad_x.view(sum.shape), grad_weight
