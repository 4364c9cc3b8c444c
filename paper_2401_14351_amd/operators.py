"""Operators on loaded weights (the last section of ``include/sllm.h``).

Matrices in microscaled 4-bit floating point (MX FP4), products with them and
token embeddings, on torch tensors in device memory:

* :func:`mx4_quantize`, :func:`mx4_dequantize`: a loaded matrix into an
  :class:`Mx4` (4.25 bits a value) and back.
* :func:`mx4_linear`: ``x @ W.T`` for one token or a whole prompt, x a tensor
  or an :class:`Mx4`; :func:`mx4_linear_grad`: ``dy @ W``.
* :func:`embedding`: scaled table rows by token, from a tensor or an
  :class:`Mx4`; :func:`embedding_grad`: the table's gradient.

Operators run on ``stream`` (by default the device's current stream) and return
without waiting.  Their outputs and workspaces belong to that stream; inputs
made on another one must be ready for it (``stream.wait_stream(...)``), and are
kept from reuse until it has passed the call.  ``mx4_linear`` and ``embedding``
take part in autograd where their input or table requires a gradient.  There is
no forward mode: a tensor with a tangent is refused.

Rows may be apart by any stride that keeps them from overlapping, but the
elements of a row must be adjacent: other tensors, broadcast ones among them, are
refused, not copied.
"""

from __future__ import annotations

import ctypes as C
import functools
from types import SimpleNamespace
from typing import Optional, Union

import torch
import torch.autograd.forward_ad as forward_ad

from paper_2401_14351_amd import binding

BLOCK = 32  # columns that share a scale

_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_ID_BITS = {torch.int32: 32, torch.int64: 64}


def _pitches(cols: int):
    blocks = -(-cols // BLOCK)
    return blocks * 16, -(-blocks // 16) * 16


class Mx4:
    """A matrix in MX FP4: ``codes`` (rows, blocks * 16) and ``scales`` (rows,
    blocks rounded up to 16), both contiguous uint8, laid out as ``sllm_mx``.
    It is those tensors, wherever their storage is when it is used."""

    __slots__ = ("_codes", "_scales", "_cols")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int):
        self._codes, self._scales, self._cols = codes, scales, cols
        self._check()

    def _check(self):
        cols = self._cols
        code_pitch, scale_pitch = _pitches(cols)
        for name, t, pitch in (("codes", self._codes, code_pitch), ("scales", self._scales, scale_pitch)):
            if t.dtype != torch.uint8 or t.dim() != 2 or t.shape[1] != pitch or not t.is_contiguous():
                raise ValueError(f"{name}: expected a contiguous uint8 tensor of {pitch} columns for {cols} columns, "
                                 f"got {t.dtype} with shape {tuple(t.shape)} and strides {t.stride()}")
        if self._codes.shape[0] != self._scales.shape[0] or self._codes.device != self._scales.device:
            raise ValueError("codes and scales differ in rows or device")

    @classmethod
    def _of(cls, codes: torch.Tensor, scales: torch.Tensor, cols: int) -> "Mx4":
        """The same without a check."""
        q = cls.__new__(cls)
        q._codes, q._scales, q._cols = codes, scales, cols
        return q

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Mx4":
        """A matrix whose contents are not set."""
        code_pitch, scale_pitch = _pitches(cols)
        return cls._of(torch.empty((rows, code_pitch), dtype=torch.uint8, device=device),
                       torch.empty((rows, scale_pitch), dtype=torch.uint8, device=device), cols)

    @classmethod
    def _beside(cls, t: torch.Tensor, rows: int, cols: int) -> "Mx4":
        """One whose contents are not set, where t is: half a microsecond less than by naming the device."""
        code_pitch, scale_pitch = _pitches(cols)
        return cls._of(t.new_empty((rows, code_pitch), dtype=torch.uint8), t.new_empty((rows, scale_pitch), dtype=torch.uint8), cols)

    def __reduce__(self):
        return Mx4, (self._codes, self._scales, self._cols)

    @property
    def _struct(self) -> binding.Mx:
        self._check()
        return binding.Mx(self._codes.data_ptr(), self._scales.data_ptr(), self.rows, self._cols)

    @property
    def codes(self) -> torch.Tensor:
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        return self._scales

    @property
    def rows(self) -> int:
        return self._codes.shape[0]

    @property
    def cols(self) -> int:
        return self._cols

    @property
    def shape(self):
        return torch.Size((self.rows, self.cols))

    @property
    def device(self):
        return self.codes.device

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()

    def __getitem__(self, rows: slice) -> "Mx4":
        """A run of rows, sharing this matrix's memory."""
        if not isinstance(rows, slice) or rows.step not in (None, 1):
            raise ValueError("an Mx4 is indexed by a run of rows")
        return Mx4(self.codes[rows], self.scales[rows], self.cols)

    def __repr__(self):
        return f"Mx4({self.rows} x {self.cols}, {self.device})"


def _matrix(t: torch.Tensor, name: str) -> binding.Matrix:
    """The rows of t (its last dimension's runs of elements)."""
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: {t.dtype} is not float32, float16 or bfloat16")
    if not t.is_cuda:
        raise ValueError(f"{name} is not in device memory")
    if t.is_neg():
        raise ValueError(f"{name} is a negated view of other elements")
    dim = t.dim()
    if dim == 0:
        raise ValueError(f"{name} has no dimensions")
    if dim > 2:
        cols = t.shape[-1]
        rows = t.numel() // cols if cols else t.shape[:-1].numel()
        if not (rows and cols):
            return binding.Matrix(t.data_ptr(), rows, cols, cols, code, 0)
        try:
            t = t.view(rows, cols)
        except RuntimeError:
            raise ValueError(f"{name}: its rows are not apart by one stride (strides {t.stride()})") from None
    strides = t.stride()
    cols = t.shape[-1]
    if cols > 1 and strides[-1] != 1:
        raise ValueError(f"{name}: the elements of a row are not adjacent (strides {strides})")
    if dim == 1:
        return binding.Matrix(t.data_ptr(), 1, cols, cols, code, 0)
    rows = t.shape[0]
    # a single row's or no row's stride says nothing
    return binding.Matrix(t.data_ptr(), rows, cols, strides[0] if rows > 1 else cols, code, 0)


def _ids(t: torch.Tensor) -> binding.Ids:
    bits = _ID_BITS.get(t.dtype)
    if bits is None:
        raise ValueError(f"tokens: {t.dtype} is not int32 or int64")
    if not t.is_cuda:
        raise ValueError("tokens are not in device memory")
    if not t.is_contiguous():
        raise ValueError(f"tokens are not contiguous (strides {t.stride()})")
    if t.is_neg():
        raise ValueError("tokens are a negated view of others")
    return binding.Ids(t.data_ptr(), t.numel(), bits, 0)


def _index(t) -> int:
    return (t._codes if isinstance(t, Mx4) else t).get_device()


def _one_device(first, *others) -> int:
    """The index of the device that all of them are on."""
    device = _index(first)
    for t in others:
        if t is not None and _index(t) != device:
            raise ValueError(f"inputs on {first.device} and {t.device}")
    return device


# torch.cuda.current_stream(device).cuda_stream without the stream object, which costs 2 us
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _on_stream(stream, operator, *args, keep=(), **kwargs):
    """Run ``operator`` with ``stream`` current: what it allocates then belongs to
    that stream, and its inputs are kept from reuse until it has passed the call."""
    device = keep[0].device
    if device.type != "cuda":
        return operator(*args, **kwargs)  # which says so
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream, device=device)
    elif stream.device != device:
        raise ValueError(f"a stream of {stream.device} for inputs on {device}")
    with torch.cuda.stream(stream):
        result = operator(*args, **kwargs)
    for t in keep:
        if t is not None:
            for u in ((t.codes, t.scales) if isinstance(t, Mx4) else (t,)):
                u.record_stream(stream)
    return result


def _refuse_tangent(t):
    # (unpack_dual looks for the level itself, in half a microsecond more)
    if getattr(forward_ad, "_current_level", 0) >= 0 and isinstance(t, torch.Tensor) \
            and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError("a tensor has a tangent: the operators have no forward mode")


def _output(out: Optional[torch.Tensor], shape, rows: int, cols: int, dtype: torch.dtype, like: torch.Tensor):
    """A result of ``rows`` x ``cols`` and its rows: ``out``, or a new tensor where ``like`` is."""
    if out is None:
        code = _DTYPE.get(dtype)
        if code is None:
            raise ValueError(f"out: {dtype} is not float32, float16 or bfloat16")
        out = like.new_empty(shape, dtype=dtype)
        return out, binding.Matrix(out.data_ptr(), rows, cols, cols, code, 0)
    if out.shape != torch.Size(shape) or out.device != like.device:
        raise ValueError(f"out: expected shape {tuple(shape)} on {like.device}, got {tuple(out.shape)} on {out.device}")
    _refuse_tangent(out)
    if out.requires_grad:
        _refuse_grad(out)
    return out, _matrix(out, "out")


def _refuse_grad(*tensors):
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError("an operator that writes to a given tensor takes no part in autograd")


def _written(out: Optional[torch.Tensor], *more: torch.Tensor):
    """Count a write to given tensors as one of torch's own in place: a backward pass that has saved them then raises."""
    for t in (out, *more):
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


def _workspace(query, *args) -> int:
    """How many bytes of workspace a call with these operands needs."""
    n = C.c_uint64()
    binding.check(query(*args, n))
    return n.value


def _call(fn, query, operands, out, device):
    """fn over its operands and output, with the workspace that the query asks for."""
    n = _workspace(query, *operands)
    if n:
        ws = torch.empty(n, dtype=torch.uint8, device=f"cuda:{device}")
        code = fn(*operands, out, ws.data_ptr(), n, device, _raw_stream(device))
    else:
        code = fn(*operands, out, None, 0, device, _raw_stream(device))
    binding.check(code)


@functools.lru_cache(maxsize=None)
def _native():
    """The extension that makes ordinary calls (tensors on one GPU whose rows need no
    second look, results allocated) and the entry points' addresses, or None
    where it was not built for this Python and torch.  Its functions return the
    result, None for a call that is not ordinary, or a failed call's code."""
    ext = binding._views_ext()
    if not hasattr(ext, "product"):
        return None
    L = binding.lib()
    names = ("sllm_mx_quantize", "sllm_mx_dequantize", "sllm_mx_linear", "sllm_mx_linear_workspace", "sllm_mx_linear_mx",
             "sllm_mx_linear_mx_workspace", "sllm_mx_linear_grad", "sllm_mx_linear_grad_workspace", "sllm_embedding",
             "sllm_embedding_mx", "sllm_embedding_grad", "sllm_embedding_grad_workspace")
    return SimpleNamespace(ext=ext, **{n[5:]: C.cast(getattr(L, n), C.c_void_p).value for n in names})


def _product(call: str, x, w, out_dtype, grad: int):
    """A product by the extension, or None."""
    native, device = _native(), x.get_device()
    code = -1 if out_dtype is None else _DTYPE.get(out_dtype)
    if native is None or device < 0 or code is None:
        return None
    y = native.ext.product(getattr(native, call), getattr(native, call + "_workspace"), x, w._codes, w._scales, w._cols, code, grad,
                           device, _raw_stream(device))
    if y.__class__ is int:
        binding.check(y)
    return y


def mx4_quantize(x: torch.Tensor, out: Optional[Mx4] = None, stream=None) -> Mx4:
    """The rows of x (its leading dimensions flattened) in MX FP4.  No gradient
    passes: an x that requires one has to be detached, or quantised under
    ``torch.no_grad()``."""
    if stream is not None:
        return _on_stream(stream, mx4_quantize, x, out, keep=(x, out))
    _refuse_tangent(x)
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError("x requires a gradient, which quantisation does not pass on")
    device = x.get_device()
    if out is None and device >= 0 and _native() is not None:
        native = _native()
        parts = native.ext.quantize(native.mx_quantize, x, device, _raw_stream(device))
        if parts.__class__ is int:
            binding.check(parts)
        if parts is not None:
            return Mx4._of(*parts, x.shape[-1])
    src = _matrix(x, "x")
    device = _one_device(x, out)
    q = Mx4._beside(x, src.rows, src.cols) if out is None else out
    if q.rows != src.rows or q.cols != src.cols:
        raise ValueError(f"out: expected {src.rows} x {src.cols}, got {q.rows} x {q.cols}")
    binding.check(binding.lib().sllm_mx_quantize(src, q._struct, device, _raw_stream(device)))
    if out is not None:
        _written(out.codes, out.scales)
    return q


def mx4_dequantize(q: Mx4, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The values q stands for, rounded to ``dtype`` (or the type of ``out``)."""
    if stream is not None:
        return _on_stream(stream, mx4_dequantize, q, dtype, out, keep=(q, out))
    device = _index(q)
    if out is None and device >= 0 and dtype in _DTYPE and _native() is not None:
        native = _native()
        y = native.ext.dequantize(native.mx_dequantize, q._codes, q._scales, q._cols, _DTYPE[dtype], device, _raw_stream(device))
        if y.__class__ is int:
            binding.check(y)
        if y is not None:
            return y
    y, rows = _output(out, (q.rows, q.cols), q.rows, q.cols, dtype, q.codes)
    binding.check(binding.lib().sllm_mx_dequantize(q._struct, rows, device, _raw_stream(device)))
    _written(out)
    return y


def mx4_linear(x: Union[torch.Tensor, Mx4], w: Mx4, out: Optional[torch.Tensor] = None,
               out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """``x @ w.T``: (..., w.rows) for x (..., w.cols).

    x as a tensor keeps its own precision; as an :class:`Mx4` both sides are in
    four bits.  The result has ``out_dtype``, by default x's type (bfloat16 for
    an :class:`Mx4`)."""
    if stream is not None:
        return _on_stream(stream, mx4_linear, x, w, out, out_dtype, keep=(x, w, out))
    if isinstance(x, Mx4):
        return _linear_mx(x, w, out, out_dtype)
    _refuse_tangent(x)
    if x.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise ValueError("an operator that writes to a given tensor takes no part in autograd")
        return _Linear.apply(x, w, out_dtype)
    return _linear(x, w, out, out_dtype)


def _linear(x, w, out, out_dtype):
    if out is None:
        y = _product("mx_linear", x, w, out_dtype, 0)
        if y is not None:
            return y
    L = binding.lib()
    src = _matrix(x, "x")
    device = _one_device(x, w)
    y, rows = _output(out, (*x.shape[:-1], w.rows), src.rows, w.rows, out_dtype or x.dtype, x)
    _call(L.sllm_mx_linear, L.sllm_mx_linear_workspace, (src, w._struct), rows, device)
    _written(out)
    return y


def _linear_mx(x, w, out, out_dtype):
    device = _one_device(x, w)
    code = _DTYPE.get(out_dtype or torch.bfloat16)
    if out is None and device >= 0 and code is not None and _native() is not None:
        native = _native()
        y = native.ext.product_mx(native.mx_linear_mx, native.mx_linear_mx_workspace, x._codes, x._scales, x._cols, w._codes,
                                  w._scales, w._cols, code, device, _raw_stream(device))
        if y.__class__ is int:
            binding.check(y)
        if y is not None:
            return y
    L = binding.lib()
    y, rows = _output(out, (x.rows, w.rows), x.rows, w.rows, out_dtype or torch.bfloat16, x.codes)
    _call(L.sllm_mx_linear_mx, L.sllm_mx_linear_mx_workspace, (x._struct, w._struct), rows, device)
    _written(out)
    return y


def mx4_linear_grad(dy: torch.Tensor, w: Mx4, out: Optional[torch.Tensor] = None,
                    out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """``dy @ w``, the gradient of :func:`mx4_linear` by x: (..., w.cols) for dy
    (..., w.rows)."""
    if stream is not None:
        return _on_stream(stream, mx4_linear_grad, dy, w, out, out_dtype, keep=(dy, w, out))
    _refuse_tangent(dy)
    _refuse_grad(dy)
    if out is None:
        dx = _product("mx_linear_grad", dy, w, out_dtype, 1)
        if dx is not None:
            return dx
    L = binding.lib()
    src = _matrix(dy, "dy")
    device = _one_device(dy, w)
    dx, rows = _output(out, (*dy.shape[:-1], w.cols), src.rows, w.cols, out_dtype or dy.dtype, dy)
    _call(L.sllm_mx_linear_grad, L.sllm_mx_linear_grad_workspace, (src, w._struct), rows, device)
    _written(out)
    return dx


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, out_dtype):
        # saved as tensors are, so that a change of the weight before the backward pass
        # raises, and hooks on what is saved see it; tensors of inference mode cannot be
        ctx.w = w if w.codes.is_inference() or w.scales.is_inference() else None
        if ctx.w is None:
            ctx.save_for_backward(w.codes, w.scales)
        ctx.cols, ctx.dtype = w.cols, x.dtype
        return _linear(x, w, None, out_dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        w = Mx4(*ctx.saved_tensors, ctx.cols) if ctx.w is None else ctx.w
        # gradients of sums and means arrive with strides of 0
        return mx4_linear_grad(dy.contiguous(), w, out_dtype=ctx.dtype), None, None


def embedding(table: Union[torch.Tensor, Mx4], tokens: torch.Tensor, scale: float = 1.0,
              out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
              stream=None) -> torch.Tensor:
    """``scale`` times the table's rows of ``tokens`` (int32 or int64): shape
    ``tokens.shape + (columns,)``, in ``out_dtype`` (by default the table's
    type, bfloat16 for an :class:`Mx4`).  A token outside the table is padding:
    a row of zeros."""
    if stream is not None:
        return _on_stream(stream, embedding, table, tokens, scale, out, out_dtype, keep=(table, tokens, out))
    _refuse_tangent(table)
    if not isinstance(table, Mx4) and table.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise ValueError("an operator that writes to a given tensor takes no part in autograd")
        return _Embedding.apply(table, tokens, scale, out_dtype)
    return _embedding(table, tokens, scale, out, out_dtype)


def _embedding(table, tokens, scale, out, out_dtype):
    device, mx = _one_device(table, tokens), isinstance(table, Mx4)
    code = (2 if mx else -1) if out_dtype is None else _DTYPE.get(out_dtype)
    if out is None and device >= 0 and code is not None and _native() is not None:
        native = _native()
        y = native.ext.lookup(native.embedding_mx if mx else native.embedding, table._codes if mx else table,
                              table._scales if mx else None, table._cols if mx else 0, tokens, scale, code, device,
                              _raw_stream(device))
        if y.__class__ is int:
            binding.check(y)
        if y is not None:
            return y
    L = binding.lib()
    ids = _ids(tokens)
    if isinstance(table, Mx4):
        fn, src, dtype = L.sllm_embedding_mx, table._struct, torch.bfloat16
    elif table.dim() == 2:
        fn, src, dtype = L.sllm_embedding, _matrix(table, "table"), table.dtype
    else:
        raise ValueError(f"table: expected rows and columns, got shape {tuple(table.shape)}")
    like = table.codes if isinstance(table, Mx4) else table
    y, rows = _output(out, (*tokens.shape, src.cols), ids.n, src.cols, out_dtype or dtype, like)
    binding.check(fn(src, ids, scale, rows, device, _raw_stream(device)))
    _written(out)
    return y


def embedding_grad(dy: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0,
                   out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                   accumulate: bool = False, stream=None) -> torch.Tensor:
    """The gradient of :func:`embedding` by a table of ``vocab`` rows: row v is
    ``scale`` times the sum of dy over the positions of token v, in their order.
    ``accumulate`` adds it to ``out`` instead of replacing its contents."""
    if stream is not None:
        return _on_stream(stream, embedding_grad, dy, tokens, vocab, scale, out, out_dtype, accumulate,
                          keep=(dy, tokens, out))
    _refuse_tangent(dy)
    _refuse_grad(dy)
    if accumulate and out is None:
        raise ValueError("accumulate needs a gradient to add to")
    if dy.shape[:-1] != tokens.shape:
        raise ValueError(f"dy of shape {tuple(dy.shape)} for tokens of shape {tuple(tokens.shape)}")
    device = _one_device(dy, tokens)
    code = -1 if out_dtype is None else _DTYPE.get(out_dtype)
    if out is None and device >= 0 and code is not None and _native() is not None:
        native = _native()
        y = native.ext.lookup_grad(native.embedding_grad, native.embedding_grad_workspace, dy, tokens, vocab, scale, code, device,
                                   _raw_stream(device))
        if y.__class__ is int:
            binding.check(y)
        if y is not None:
            return y
    L = binding.lib()
    ids, src = _ids(tokens), _matrix(dy, "dy")
    g, grad = _output(out, (vocab, src.cols), vocab, src.cols, out_dtype or dy.dtype, dy)
    n = _workspace(L.sllm_embedding_grad_workspace, ids.n, grad)
    ws = torch.empty(n, dtype=torch.uint8, device=dy.device) if n else None
    binding.check(L.sllm_embedding_grad(src, ids, scale, 1 if accumulate else 0, grad, ws.data_ptr() if n else None, n,
                                        device, _raw_stream(device)))
    _written(out)
    return g


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, out_dtype):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.dtype, ctx.scale = table.shape[0], table.dtype, scale
        return _embedding(table, tokens, scale, None, out_dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        (tokens,) = ctx.saved_tensors
        return embedding_grad(dy.contiguous(), tokens, ctx.vocab, ctx.scale, out_dtype=ctx.dtype), None, None, None
