"""Microscaled 4-bit matrices: quantisation and products.

Argument marshalling for the rrf_mx4_* entry points (include/rrf.h), which
describe the layout and the arithmetic.  Real matrices are column-major, as
everywhere in this package (``colmajor``).
"""

import ctypes

from . import _abi
from .ortho import _torch, no_graph, on_device, real_code

BLOCK = 32    # rows that share a scale
PAD = 256     # a column is padded to a multiple of this


def _padded(k):
    return -(-k // PAD) * PAD


class Mx4:
    """A k x n matrix in 4 bits: codes (n x kp/2) and scales (n x kp/32), uint8,
    contiguous, kp the next multiple of 256.  ``A[a:b]`` is a range of columns."""

    def __init__(self, codes, scales, k):
        torch = _torch()
        kp = _padded(k)
        for name, t, width in (("codes", codes, kp // 2), ("scales", scales, kp // BLOCK)):
            if t.dtype != torch.uint8 or t.dim() != 2:
                raise TypeError(f"{name} must be a 2-D uint8 tensor")
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous CUDA tensor")
            if t.shape[1] != width:
                raise ValueError(f"{name} needs {width} bytes a column for {k} rows")
        if codes.shape[0] != scales.shape[0] or codes.device != scales.device:
            raise ValueError("codes and scales differ in columns or device")
        self._buffer, self._codes, self._scales = None, codes, scales
        self.k, self.n, self.device = k, codes.shape[0], codes.device

    @classmethod
    def _empty(cls, k, n, device):
        """Codes and scales one after the other in one allocation, cut into the
        two tensors where they are asked for: small calls are bound by the host
        (quantising one column of 11008: 9.6 -> 7.2 us)."""
        self = cls.__new__(cls)
        kp = _padded(k)
        self._buffer = _torch().empty(n * (kp // 2 + kp // BLOCK), dtype=_torch().uint8, device=device)
        self._codes = self._scales = None
        self.k, self.n, self.device = k, n, device
        return self

    def _cut(self):
        kp = _padded(self.k)
        end = self.n * (kp // 2)
        self._codes = self._buffer[:end].view(self.n, kp // 2)
        self._scales = self._buffer[end:].view(self.n, kp // BLOCK)

    @property
    def codes(self):
        if self._codes is None:
            self._cut()
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._cut()
        return self._scales

    @property
    def _memory(self):
        """The tensors that hold it."""
        return (self._codes, self._scales) if self._buffer is None else (self._buffer,)

    def _addresses(self):
        if self._buffer is None:
            return self._codes.data_ptr(), self._scales.data_ptr()
        at = self._buffer.data_ptr()
        return at, at + self.n * (_padded(self.k) // 2)

    @property
    def shape(self):
        return (self.k, self.n)

    def __getitem__(self, cols):
        if not isinstance(cols, slice) or cols.step not in (None, 1):
            raise TypeError("only a range of columns can be taken")
        return Mx4(self.codes[cols], self.scales[cols], self.k)

    def dequantize(self, dtype=None, stream=None):
        """The values (k x n, column-major), float32 unless given."""
        torch = _torch()
        dtype = torch.float32 if dtype is None else dtype
        code = real_code(dtype)
        with on_device(*_first(self._memory, stream)) as s:
            out = _columns(self.k, self.n, dtype, self.device)
            _abi.check(_abi.load().rrf_mx4_dequantize(
                code, self.k, self.n, *self._addresses(),
                out.data_ptr(), max(self.k, 1), s.handle), "rrf_mx4_dequantize")
        return out


def _first(tensors, stream):
    """Arguments of on_device for some tensors."""
    return (tensors[0], stream, *tensors[1:])


def _columns(rows, cols, dtype, device):
    """A new column-major matrix."""
    return _torch().empty_strided((rows, cols), (1, max(rows, 1)), dtype=dtype, device=device)


def _colmajor_ld(t, name):
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a 2-D CUDA tensor")
    rows, cols = t.shape
    ld = t.stride(1) if cols > 1 else max(1, rows)
    if (rows > 1 and t.numel() and t.stride(0) != 1) or ld < max(1, rows):
        raise ValueError(f"{name} must be column-major (use colmajor())")
    return ld


def mx4_quantize(X, stream=None):
    """X (k x n, column-major; float32, bfloat16 or float16) in 4 bits, which
    carry no gradient."""
    torch = _torch()
    code = real_code(X.dtype)
    ldx = _colmajor_ld(X, "X")
    k, n = X.shape
    with on_device(X, stream) as s:
        A = Mx4._empty(k, n, X.device)
        _abi.check(_abi.load().rrf_mx4_quantize(
            code, k, n, X.data_ptr(), ldx, *A._addresses(), s.handle), "rrf_mx4_quantize")
    return A


def mx4_product(A, B, dtype=None, stream=None):
    """A^T B of two 4-bit matrices with the same number of rows (A.n x B.n,
    column-major, float32 unless given)."""
    torch = _torch()
    dtype = torch.float32 if dtype is None else dtype
    code = real_code(dtype)
    if A.k != B.k:
        raise ValueError("A and B differ in rows")
    if A.device != B.device:
        raise ValueError("A and B are on different devices")
    with on_device(*_first(A._memory + B._memory, stream)) as s:
        C = _columns(A.n, B.n, dtype, A.device)
        _abi.check(_abi.load().rrf_mx4_product(
            code, A.n, B.n, A.k, *A._addresses(), *B._addresses(), C.data_ptr(), max(A.n, 1),
            s.handle), "rrf_mx4_product")
    return C


_sizes = {}     # workspace bytes by (type, trans, k, m, n)


def _apply_workspace(*key):
    got = _sizes.get(key)
    if got is None:
        out = ctypes.c_size_t()
        _abi.check(_abi.load().rrf_mx4_apply_workspace(*key, ctypes.byref(out)),
                   "rrf_mx4_apply_workspace")
        if len(_sizes) >= 4096:
            _sizes.clear()
        got = _sizes[key] = out.value
    return got


def mx4_apply(A, B, trans=True, stream=None):
    """A^T B (trans) or A B of a 4-bit matrix A and a real column-major B, in
    B's type.  ``mx4_apply(A, dC, trans=not t)`` is the gradient for B of
    ``C = mx4_apply(A, B, trans=t)``; autograd does not record it, and a B that
    requires grad is refused outside torch.no_grad()."""
    torch = _torch()
    code = real_code(B.dtype)
    no_graph("B", B)
    ldb = _colmajor_ld(B, "B")
    if A.device != B.device:
        raise ValueError("A and B are on different devices")
    if B.shape[0] != (A.k if trans else A.n):
        raise ValueError("A and B do not chain")
    rows, n = A.n if trans else A.k, B.shape[1]
    with on_device(B, stream, *A._memory) as s:
        C = _columns(rows, n, B.dtype, B.device)
        need = _apply_workspace(code, 1 if trans else 0, A.k, A.n, n)
        ws = torch.empty(need, dtype=torch.uint8, device=B.device) if need else None
        _abi.check(_abi.load().rrf_mx4_apply(
            code, 1 if trans else 0, A.k, A.n, *A._addresses(), B.data_ptr(), ldb, n, C.data_ptr(),
            max(rows, 1), ws.data_ptr() if need else None, need, s.handle), "rrf_mx4_apply")
    return C
