"""Binding of the playback operators (include/peat_ops.h), and a linear layer made of them.

``peat_quantize_i8`` and ``peat_matmul_i8`` (in one call: ``peat_product_i8``)
are a linear layer's products in 8-bit integers with a scale for each row of
either operand; ``peat_grad_norm`` and ``peat_grad_clip`` the norm over a list
of gradient tensors and their clipping.  As in the rest of the binding, a ``_raw`` function fills outputs
that the caller holds; the plain ones allocate them.  All of them only enqueue
work on the stream (``peat_grad_norm`` and ``peat_grad_clip``, which return
host numbers, wait for it).

``Linear8`` is the layer as a playback step replays it (Alg. 1's Fwd, InGrad
and WgGrad at a lower precision): the weight held in 8 bits, the recorded
tensors rounded on the way in.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import Optional, Sequence

OUT_I32 = 100
GRADNORM_BYTES = 16
NORM_TYPES = {"2": 0, "1": 1, "inf": 2}
BAD_MODES = {"propagate": 0, "zero": 1, "keep": 2}

OPS_EXPORTS = ("peat_quantize_i8", "peat_matmul_i8", "peat_product_i8", "peat_grad_norm", "peat_grad_clip")
INT8 = 101


class GradEntry(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class Operand8(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("axis", ctypes.c_int32)]


def register(L) -> None:
    """Argument types of the entry points in a loaded library."""
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    L.peat_quantize_i8.argtypes = [vp, vp, i64, i64, i64, i32, i32, vp, i64, vp, vp, i64, vp]
    L.peat_matmul_i8.argtypes = [vp, vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, vp, i64, i32, vp]
    op = ctypes.POINTER(Operand8)
    L.peat_product_i8.argtypes = [vp, op, op, vp, vp, i64, i32, vp]
    L.peat_grad_norm.argtypes = [vp, vp, i64, i32, f32, vp, vp, vp]
    L.peat_grad_clip.argtypes = [vp, vp, i64, i32, f32, f32, f32, i32, vp, vp, vp]
    for name in OPS_EXPORTS:
        getattr(L, name).restype = i32


_entry = {}


def _call(h, name, *args) -> None:
    f = _entry.get(name)
    if f is None:
        from . import load
        f = _entry[name] = getattr(load(), name)
    rc = f(h.ptr, *args)
    if rc:
        from . import _check
        _check(rc, h)


_raw_stream = None


def _stream(h, stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    global _raw_stream
    if _raw_stream is None:
        import torch
        # the current stream's handle without a Stream object around it (1 us less a call), where torch has it
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream(h.device)


_NOTHING = contextlib.nullcontext()


def _on(stream):
    """Allocations belong to the stream that the call runs on."""
    if stream is None:
        return _NOTHING
    import torch
    return torch.cuda.stream(stream)


_codes = {}  # by torch type; filled by the first use (an import of torch within each call would take 0.3 us)


def _code_or_int8(t) -> Optional[int]:
    """A tensor's type code, INT8's among them; None for other types."""
    c = _codes.get(t.dtype)
    if c is None and not _codes:
        import torch
        _codes.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.int8: INT8, torch.int32: OUT_I32})
        c = _codes.get(t.dtype)
    return c if c != OUT_I32 else None


def _code(t) -> int:
    c = _code_or_int8(t)
    if c is None or c == INT8:
        raise TypeError(f"unsupported dtype {t.dtype}: float32, float16 or bfloat16")
    return c


def _is_int32(t) -> bool:
    _code_or_int8(t)
    return _codes.get(t.dtype) == OUT_I32


def _matrix(h, t, name: str) -> int:
    """The row distance of a matrix whose rows are contiguous, on the handle's device."""
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    if t.get_device() != h.device:
        raise ValueError(f"{name} must be a CUDA tensor on the handle's device")
    rows, cols = t.shape
    s0, s1 = t.stride()
    if s1 != 1 and cols > 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    if rows <= 1:
        return cols
    if s0 < cols:
        raise ValueError(f"the rows of {name} overlap")
    return s0


def _vector(h, t, n: int, name: str) -> Optional[int]:
    if t is None:
        return None
    if _code_or_int8(t) != 0 or t.numel() != n or not t.is_contiguous() or t.get_device() != h.device:
        raise ValueError(f"{name} must be a contiguous float32 tensor of {n} elements on the handle's device")
    return t.data_ptr()


def _padded(rows: int, cols: int, device):
    """An int8 matrix whose rows start on 16-byte boundaries, as the products read them fastest."""
    import torch
    return torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=device)[:, :cols]


def peat_quantize_i8_raw(h, x, axis: int, q=None, scale=None, values=None, stream=None) -> None:
    """peat_quantize_i8 on preallocated device outputs: q int8 (axis 0: x's shape, axis 1: transposed), scale
    float32 [rows or cols], values (x's shape and type); each may be None, but not both of q and values."""
    ldx = _matrix(h, x, "x")
    rows, cols = x.shape
    ldq = ldv = 0
    if q is not None:
        ldq = _matrix(h, q, "q")
        if _code_or_int8(q) != INT8 or tuple(q.shape) != ((rows, cols) if axis == 0 else (cols, rows)):
            raise ValueError("q must be int8 of x's shape (axis 0) or its transpose (axis 1)")
    if values is not None:
        ldv = _matrix(h, values, "values")
        if values.dtype != x.dtype or values.shape != x.shape:
            raise ValueError("values must have x's shape and type")
    _call(h, "peat_quantize_i8", x.data_ptr(), rows, cols, ldx, _code(x), axis, None if q is None else q.data_ptr(),
          ldq, _vector(h, scale, cols if axis else rows, "scale"), None if values is None else values.data_ptr(), ldv,
          _stream(h, stream))


def peat_quantize_i8(h, x, axis: int = 0, stream=None):
    """x as 8-bit integers with a scale for each row (axis 0) or column (axis 1): (q, scale), for axis 1 q
    transposed.  q's rows are padded to 16 bytes (a view)."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must have two dimensions")
    rows, cols = x.shape if axis == 0 else (x.shape[1], x.shape[0])
    with _on(stream):
        q = _padded(rows, cols, x.device)
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
        peat_quantize_i8_raw(h, x, axis, q, scale, None, stream)
    return q, scale


def peat_matmul_i8_raw(h, a, a_scale, b, b_scale, out, bias=None, stream=None) -> None:
    """peat_matmul_i8 into out [M, N] (float32, float16, bfloat16, or int32 for the sums themselves) from a [M, K]
    and b [N, K] int8 with their scales (None: 1)."""
    lda, ldb, ldo = _matrix(h, a, "a"), _matrix(h, b, "b"), _matrix(h, out, "out")
    (M, K), N = a.shape, b.shape[0]
    if _code_or_int8(a) != INT8 or _code_or_int8(b) != INT8:
        raise TypeError("a and b must be int8")
    if b.shape[1] != K:
        raise ValueError("a and b differ in their row length")
    if tuple(out.shape) != (M, N):
        raise ValueError("out must be [rows of a, rows of b]")
    _call(h, "peat_matmul_i8", a.data_ptr(), lda, _vector(h, a_scale, M, "a_scale"), b.data_ptr(), ldb,
          _vector(h, b_scale, N, "b_scale"), _vector(h, bias, N, "bias"), M, N, K, out.data_ptr(), ldo,
          OUT_I32 if _is_int32(out) else _code(out), _stream(h, stream))


def peat_matmul_i8(h, a, a_scale, b, b_scale, bias=None, out_dtype=None, stream=None):
    """(sum over k of a[m, k] b[n, k]) a_scale[m] b_scale[n] + bias[n] as out_dtype (float32 unless given)."""
    import torch
    with _on(stream):
        out = torch.empty(a.shape[0], b.shape[0], dtype=out_dtype or torch.float32, device=a.device)
        peat_matmul_i8_raw(h, a, a_scale, b, b_scale, out, bias, stream)
    return out


def _operand(h, t, axis: int, scale, name: str):
    """(structure, rows of the operand, its K) of a matrix that is 8-bit integers or is rounded to them."""
    ld = _matrix(h, t, name)
    rows, cols = t.shape
    code = _code_or_int8(t)
    if code == INT8:
        if axis != 0:
            raise ValueError(f"{name} is integers already: axis 0")
        return Operand8(t.data_ptr(), _vector(h, scale, rows, name + "'s scale"), rows, cols, ld, INT8, 0), rows, cols
    if scale is not None:
        raise ValueError(f"{name} is not integers: it has no scale yet")
    op = Operand8(t.data_ptr(), None, rows, cols, ld, _code(t), axis)
    return (op, cols, rows) if axis else (op, rows, cols)


def _operands(h, a, b, a_axis: int, b_axis: int, a_scale, b_scale):
    """The structures of both operands, and M and N."""
    x, M, K = _operand(h, a, a_axis, a_scale, "a")
    y, N, K2 = _operand(h, b, b_axis, b_scale, "b")
    if K != K2:
        raise ValueError("a and b differ in their row length")
    return x, y, M, N


def peat_product_i8_raw(h, a, b, out, a_axis: int = 0, b_axis: int = 0, a_scale=None, b_scale=None, bias=None,
                        stream=None) -> None:
    """peat_product_i8 into out [M, N] (float32, float16 or bfloat16): each operand int8 with its scale, or a float
    matrix that is rounded with a scale for each row (axis 0) or column (axis 1; its transpose is the operand)."""
    x, y, M, N = _operands(h, a, b, a_axis, b_axis, a_scale, b_scale)
    ldo = _matrix(h, out, "out")
    if out.shape[0] != M or out.shape[1] != N:
        raise ValueError("out must be [rows of a, rows of b]")
    _call(h, "peat_product_i8", ctypes.byref(x), ctypes.byref(y), _vector(h, bias, N, "bias"), out.data_ptr(), ldo,
          _code(out), _stream(h, stream))


def peat_product_i8(h, a, b, a_axis: int = 0, b_axis: int = 0, a_scale=None, b_scale=None, bias=None, out_dtype=None,
                    stream=None):
    """The product as a new tensor of out_dtype (float32 unless given)."""
    if stream is not None:
        with _on(stream):
            return peat_product_i8(h, a, b, a_axis, b_axis, a_scale, b_scale, bias, out_dtype)
    import torch
    x, y, M, N = _operands(h, a, b, a_axis, b_axis, a_scale, b_scale)
    out = torch.empty(M, N, dtype=out_dtype or torch.float32, device=a.device)
    _call(h, "peat_product_i8", ctypes.byref(x), ctypes.byref(y), _vector(h, bias, N, "bias"), out.data_ptr(), N,
          _code(out), _stream(h, None))
    return out


class GradList:
    """A list of gradient tensors (and, for clipping, of as many output tensors; None: in place), made once and
    passed to every peat_grad_norm or peat_grad_clip.  It holds the tensors: where a program gives a parameter a
    new gradient tensor, it makes a new list."""

    def __init__(self, tensors: Sequence, outs: Optional[Sequence] = None):
        import torch
        self.tensors = list(tensors)
        self.outs = self.tensors if outs is None else list(outs)
        if len(self.outs) != len(self.tensors):
            raise ValueError("as many outputs as tensors are needed")
        self.entries = (GradEntry * max(len(self.tensors), 1))()
        self.device = self.tensors[0].device if self.tensors else None
        for i, (t, o) in enumerate(zip(self.tensors, self.outs)):
            code = _code(t)
            if not t.is_cuda or t.device != self.device or o.device != self.device:
                raise ValueError("gradients and outputs must be CUDA tensors on one device")
            if o.dtype != t.dtype or o.shape != t.shape:
                raise ValueError("an output differs from its gradient in type or shape")
            # (by order in memory: the strides of dimensions of size 1 tell nothing)
            same = t.is_contiguous() and o.is_contiguous()
            if not same and t.dim() == 4:
                same = all(v.is_contiguous(memory_format=torch.channels_last) for v in (t, o))
            if not same:
                raise ValueError("gradients must be contiguous (or channels-last), outputs of the same layout")
            self.entries[i] = GradEntry(t.data_ptr(), o.data_ptr(), t.numel(), code, 0)

    def __len__(self) -> int:
        return len(self.tensors)


def _grad_args(h, grads, record, norms):
    import torch
    if not isinstance(grads, GradList):
        grads = GradList(grads)
    if grads.device is not None and grads.device.index != h.device:
        raise ValueError("the gradients must be on the handle's device")
    if record.nbytes < GRADNORM_BYTES or not record.is_contiguous() or record.get_device() != h.device:
        raise ValueError("record must be a contiguous CUDA tensor of 16 bytes on the handle's device")
    if norms is not None and (norms.dtype != torch.float32 or norms.numel() < len(grads)):
        raise ValueError("norms must be float32, one element for each tensor")
    return grads, None if norms is None else _vector(h, norms, norms.numel(), "norms")


def peat_grad_norm_raw(h, grads, record, norms=None, norm_type: str = "2", unscale: float = 1.0, stream=None) -> None:
    """peat_grad_norm of a GradList (or a list of tensors) into record (16 bytes: float32 norm, float32 1, uint64
    count of NaN and infinite elements) and norms (float32, one a tensor, or None)."""
    grads, np_ = _grad_args(h, grads, record, norms)
    _call(h, "peat_grad_norm", grads.entries, len(grads), NORM_TYPES[norm_type], unscale, record.data_ptr(), np_,
          _stream(h, stream))


def peat_grad_clip_raw(h, grads, max_norm: float, record, norms=None, norm_type: str = "2", unscale: float = 1.0,
                       eps: float = 1e-6, bad: str = "propagate", stream=None) -> None:
    """peat_grad_clip of a GradList (or, in place, of a list of tensors); record and norms as in peat_grad_norm_raw,
    record's second float32 the clipping factor."""
    grads, np_ = _grad_args(h, grads, record, norms)
    _call(h, "peat_grad_clip", grads.entries, len(grads), NORM_TYPES[norm_type], unscale, max_norm, eps,
          BAD_MODES[bad], record.data_ptr(), np_, _stream(h, stream))


def _grad_record(record, norms, stream) -> dict:
    from . import _sync
    import torch
    _sync(stream)
    r = record.cpu()
    f = r.view(torch.float32)
    return {"norm": f[0].item(), "coef": f[1].item(), "n_bad": r.view(torch.int64)[1].item(),
            "norms": norms.cpu().numpy()}


def _grad_outputs(h, grads):
    import torch
    dev = torch.device("cuda", h.device)
    return (torch.empty(GRADNORM_BYTES, dtype=torch.uint8, device=dev),
            torch.empty(len(grads), dtype=torch.float32, device=dev))


def peat_grad_norm(h, grads, norm_type: str = "2", unscale: float = 1.0, stream=None) -> dict:
    """Norm of unscale * g over all tensors: dict of norm, n_bad (NaN and infinite elements), coef (1) and norms
    (numpy float32, one a tensor); synchronises."""
    with _on(stream):
        record, norms = _grad_outputs(h, grads)
        peat_grad_norm_raw(h, grads, record, norms, norm_type, unscale, stream)
        return _grad_record(record, norms, stream)


def peat_grad_clip(h, grads, max_norm: float, norm_type: str = "2", unscale: float = 1.0, eps: float = 1e-6,
                   bad: str = "propagate", stream=None) -> dict:
    """Scales the tensors by unscale * min(1, max_norm / (norm + eps)), in place or into the GradList's outputs;
    the dict of peat_grad_norm with the factor as coef; synchronises."""
    with _on(stream):
        record, norms = _grad_outputs(h, grads)
        peat_grad_clip_raw(h, grads, max_norm, record, norms, norm_type, unscale, eps, bad, stream)
        return _grad_record(record, norms, stream)


def _as_rows(t, K: int):
    """t [..., K] as a matrix with rows of their own: t, a view of it or, where its strides are others (transposed or
    expanded tensors), a copy."""
    x = t if t.dim() == 2 else t.reshape(t.shape[:-1].numel(), K)
    s0, s1 = x.stride()
    return x if (s1 == 1 or K <= 1) and (s0 >= K or x.shape[0] <= 1) else x.contiguous()


class Linear8:
    """y = x w^T with w [out, in] held in 8-bit integers, by row for the forward product and by column for the
    input gradient; x and the output gradient are rounded as they come (by row, or, for the weight gradient, by
    column).  Inputs are float32, float16 or bfloat16 with any leading dimensions and strides; the layer keeps none of
    them."""

    def __init__(self, h, weight, stream=None):
        self.h = h
        self.out_features, self.in_features = weight.shape
        with _on(stream):
            weight = _as_rows(weight, self.in_features)
        self.q, self.scale = peat_quantize_i8(h, weight, 0, stream)
        self.qt, self.scale_t = peat_quantize_i8(h, weight, 1, stream)
        self._w = _operand(h, self.q, 0, self.scale, "weight")
        self._wt = _operand(h, self.qt, 0, self.scale_t, "weight")

    def _product(self, t, w, name: str, bias=None, stream=None):
        """t [..., K] by row times a weight operand -> [..., N] of t's type."""
        if stream is not None:
            with _on(stream):
                return self._product(t, w, name, bias)
        import torch
        op, N, K = w
        shape = t.shape
        if not shape or shape[-1] != K:
            raise ValueError(f"the last dimension of {name} must be {K}")
        x = _as_rows(t, K)
        a, M, _ = _operand(self.h, x, 0, None, name)
        out = torch.empty((M, N), dtype=x.dtype, device=x.device)
        _call(self.h, "peat_product_i8", ctypes.byref(a), ctypes.byref(op), _vector(self.h, bias, N, "bias"),
              out.data_ptr(), N, _code(out), _stream(self.h, None))
        return out if len(shape) == 2 else out.view(*shape[:-1], N)

    def forward(self, x, bias=None, stream=None):
        """x [..., in] -> [..., out] of x's type."""
        return self._product(x, self._w, "x", bias, stream)

    def input_grad(self, grad, stream=None):
        """dL/dx [..., in] of grad's type from grad = dL/dy [..., out]."""
        return self._product(grad, self._wt, "grad", None, stream)

    def weight_grad(self, grad, x, stream=None):
        """dL/dw [out, in] in float32 from grad [..., out] and x [..., in]."""
        if stream is not None:
            with _on(stream):
                return self.weight_grad(grad, x)
        if grad.shape[-1:] != (self.out_features,) or x.shape[-1:] != (self.in_features,):
            raise ValueError(f"the last dimensions of grad and x must be {self.out_features} and {self.in_features}")
        g, x = _as_rows(grad, self.out_features), _as_rows(x, self.in_features)
        if g.shape[0] != x.shape[0]:
            raise ValueError("grad and x differ in their leading dimensions")
        return peat_product_i8(self.h, g, x, 1, 1)

    def backward(self, grad, x, stream=None):
        """(dL/dx, dL/dw)."""
        return self.input_grad(grad, stream), self.weight_grad(grad, x, stream)
