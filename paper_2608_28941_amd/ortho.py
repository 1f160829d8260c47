"""Orthogonalised updates: Newton-Schulz iteration and the step around it.

Argument marshalling for rrf_orthogonalize and rrf_muon_step (include/rrf.h).
Matrices are column-major (strides (1, ld)) or row-major (strides (ld, 1)); a
batch is a 3-D tensor of such matrices.  A row-major matrix is the transpose of
a column-major one, and the iteration commutes with transposition.
"""

import ctypes

from . import _abi
from ._abi import RRF_BF16, RRF_F16, RRF_F32

# The quintic of the Muon optimiser, five equal steps: x -> a x + b x^3 + c x^5
# takes singular values in (0, 1] to the neighbourhood of 1.
MUON_COEFFS = ((3.4445, -4.7750, 2.0315),) * 5

_sizes = {}     # workspace bytes by (type, m, n, batch, momentum)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def real_code(dt):
    """rrf_dtype of the types that these operators take."""
    torch = _torch()
    if dt == torch.float32:
        return RRF_F32
    if dt == torch.bfloat16:
        return RRF_BF16
    if dt == torch.float16:
        return RRF_F16
    raise TypeError("only float32, bfloat16 and float16 are supported")


def no_graph(name, t):
    """Refuses a tensor whose gradient the caller expects autograd to take: the
    call records none."""
    if t.requires_grad and _torch().is_grad_enabled():
        raise RuntimeError(f"{name} requires grad, which this call does not record: "
                           "detach it, or call under torch.no_grad()")


def written(*tensors):
    """Tells autograd that a call wrote them, so that a graph which kept one of
    them for its backward refuses to use it."""
    for t in tensors:
        if not t.is_inference():
            _torch().autograd.graph.increment_version(t)


class _OnDevice:
    """A tensor's device and the given stream for the time of a call;
    ``handle`` is the stream's."""

    def __init__(self, t, stream):
        torch = _torch()
        if not t.is_cuda:
            raise ValueError("expected CUDA tensors")
        if stream is not None:
            if stream.device != t.device:
                raise ValueError("the stream is another device's")
            self.guard = torch.cuda.stream(stream)
        else:
            self.guard = torch.cuda.device(t.device)
            stream = torch.cuda.current_stream(t.device)
        self.handle = stream.cuda_stream

    def __enter__(self):
        self.guard.__enter__()
        return self

    def __exit__(self, *exc):
        self.guard.__exit__(*exc)


class _Current:
    """The current device with its current stream: nothing to switch."""

    __slots__ = ("handle",)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        pass


def on_device(t, stream, *others):
    """Context of a call on t's device and the given stream (None: its current
    one), with the stream's ``handle``.  The memory of t and the others, which
    the call reads or writes, is not given away before the given stream is
    done with it.  The usual case, the current device and no stream given, is
    kept cheap: small calls are bound by the host."""
    if stream is None and t.is_cuda:
        torch = _torch()
        index = t.device.index
        if index == torch.cuda.current_device():
            c = _Current()
            c.handle = torch._C._cuda_getCurrentRawStream(index)
            return c
    context = _OnDevice(t, stream)
    if stream is not None:
        for x in (t, *others):
            x.record_stream(stream)
    return context


def _orders(t):
    """The orders that the last two strides fit: 'c' (column-major) and 'r'
    (row-major); both for a single row or column without gaps."""
    rows, cols = t.shape[-2:]
    r, c = t.stride(-2), t.stride(-1)
    fits = ""
    if (rows <= 1 or r == 1) and (cols <= 1 or c >= max(1, rows)):
        fits += "c"
    if (cols <= 1 or c == 1) and (rows <= 1 or r >= max(1, cols)):
        fits += "r"
    return fits


def _matrix(t, order):
    """(m, n, batch, ld, stride) of a matrix or batch in the given order."""
    rows, cols = t.shape[-2:]
    batch = t.shape[0] if t.dim() == 3 else 1
    if order == "c":
        m, n, ld = rows, cols, t.stride(-1) if cols > 1 else max(1, rows)
    else:
        m, n, ld = cols, rows, t.stride(-2) if rows > 1 else max(1, cols)
    return m, n, batch, ld, t.stride(0) if t.dim() == 3 else 0


def _common_order(tensors):
    fits = "cr"
    first = tensors[0][1]
    for name, t in tensors:
        if t.dim() not in (2, 3):
            raise ValueError(f"{name} must be a matrix or a batch of matrices")
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        if t.device != first.device:
            raise ValueError(f"{name} is on another device")
        if t.shape != first.shape:
            raise ValueError(f"{name}'s shape differs from {tensors[0][0]}'s")
        own = _orders(t)
        if not own:
            raise ValueError(f"{name} must be column-major or row-major")
        fits = "".join(o for o in fits if o in own)
        if not fits:
            raise ValueError(f"{name}'s order differs from the others'")
    return fits[0]


def _coeffs(coeffs):
    """(C array, steps) of a sequence of (a, b, c)."""
    steps = [[float(v) for v in abc] for abc in coeffs]
    if any(len(abc) != 3 for abc in steps):
        raise ValueError("coeffs is a list of (a, b, c)")
    flat = [v for abc in steps for v in abc]
    return (ctypes.c_double * max(1, len(flat)))(*flat), len(steps)


def orthogonalize_workspace(dtype, m, n, batch=1, momentum=False):
    """Device bytes that a call on m x n matrices needs."""
    key = (dtype, m, n, batch, momentum)
    got = _sizes.get(key)
    if got is None:
        out = ctypes.c_size_t()
        _abi.check(_abi.load().rrf_orthogonalize_workspace(
            real_code(dtype), m, n, batch, 1 if momentum else 0, ctypes.byref(out)),
            "rrf_orthogonalize_workspace")
        if len(_sizes) >= 4096:
            _sizes.clear()
        got = _sizes[key] = out.value
    return got


def _given(workspace, device):
    """The caller's workspace, checked, as a tuple; empty without one."""
    if workspace is None:
        return ()
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor")
    if workspace.device != device:
        raise ValueError("workspace is on another device")
    return (workspace,)


def _space(need, workspace, device):
    if workspace is not None:
        return workspace
    return _torch().empty(max(need, 256), dtype=_torch().uint8, device=device)


def orthogonalize(G, coeffs=MUON_COEFFS, eps=1e-7, out=None, workspace=None, stream=None):
    """Newton-Schulz iteration on G (a matrix, or a 3-D batch of them).

    X = G / (||G||_F + eps), then X <- (a I + b A + c A^2) X with A = X X^T
    for each (a, b, c) of coeffs, in float32, bfloat16 or float16.  Returns
    out (new unless given; out may be G) in G's order.  A matrix whose norm is
    not finite gives NaN throughout.  workspace: optional contiguous CUDA
    tensor of at least orthogonalize_workspace(...) bytes, 256-byte aligned.
    Asynchronous on the stream (None: the current one).  Autograd records
    nothing: a G or out that requires grad is refused outside torch.no_grad().
    """
    torch = _torch()
    code = real_code(G.dtype)
    no_graph("G", G)
    given = out is not None
    if given:
        no_graph("out", out)
    if out is None:
        order = _common_order([("G", G)])
        with on_device(G, stream):
            if order == "c":
                out = torch.empty_like(G.transpose(-1, -2), memory_format=torch.contiguous_format).transpose(-1, -2)
            else:
                out = torch.empty_like(G, memory_format=torch.contiguous_format)
    else:
        if out.dtype != G.dtype:
            raise TypeError("out's dtype differs from G's")
        order = _common_order([("G", G), ("out", out)])
    m, n, batch, ldg, sg = _matrix(G, order)
    _, _, _, ldo, so = _matrix(out, order)
    c, steps = _coeffs(coeffs)
    with on_device(G, stream, out, *_given(workspace, G.device)) as s:
        need = orthogonalize_workspace(G.dtype, m, n, batch)
        ws = _space(need, workspace, G.device)
        _abi.check(_abi.load().rrf_orthogonalize(
            code, m, n, batch, G.data_ptr(), ldg, sg, out.data_ptr(), ldo, so, c, steps,
            float(eps), ws.data_ptr(), ws.numel() * ws.element_size(), s.handle),
            "rrf_orthogonalize")
    if given:
        written(out)
    return out


def muon_step(W, M, G, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale=1.0,
              coeffs=MUON_COEFFS, eps=1e-7, workspace=None, stream=None):
    """One optimiser step on the weights W, in place:

        M <- momentum M + G
        U  = G + momentum M  (nesterov)  or  M
        W <- (1 - lr weight_decay) W - lr scale orthogonalize(U)

    W and G share a type (float32, bfloat16 or float16), the momentum M is
    float32; all three have the same shape and order.  Autograd records
    nothing, as in every optimiser step, and W may require grad; a graph that
    kept W or M for its backward refuses to use them afterwards.
    """
    code = real_code(G.dtype)
    if W.dtype != G.dtype:
        raise TypeError("W's dtype differs from G's")
    if M.dtype != _torch().float32:
        raise TypeError("the momentum M must be float32")
    order = _common_order([("W", W), ("M", M), ("G", G)])
    m, n, batch, ldw, sw = _matrix(W, order)
    _, _, _, ldm, sm = _matrix(M, order)
    _, _, _, ldg, sg = _matrix(G, order)
    c, steps = _coeffs(coeffs)
    with on_device(W, stream, M, G, *_given(workspace, G.device)) as s:
        need = orthogonalize_workspace(G.dtype, m, n, batch, True)
        ws = _space(need, workspace, W.device)
        _abi.check(_abi.load().rrf_muon_step(
            code, m, n, batch, W.data_ptr(), ldw, sw, M.data_ptr(), ldm, sm, G.data_ptr(), ldg, sg,
            float(lr), float(momentum), 1 if nesterov else 0, float(weight_decay), float(scale),
            c, steps, float(eps), ws.data_ptr(), ws.numel() * ws.element_size(), s.handle),
            "rrf_muon_step")
    written(W, M)
    return W
