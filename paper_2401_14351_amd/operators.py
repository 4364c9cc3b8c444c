"""Operators on loaded weights (the last section of ``include/sllm.h``).

Matrices in microscaled 4-bit floating point (MX FP4), products with them, token
embeddings, and the norms and attention between them, on torch tensors in device
memory:

* :func:`mx4_quantize`, :func:`mx4_dequantize`: a loaded matrix into an
  :class:`Mx4` (4.25 bits a value) and back.
* :func:`mx4_linear`: ``x @ W.T`` for one token or a whole prompt, x a tensor
  or an :class:`Mx4`; :func:`mx4_linear_grad`: ``dy @ W``.
* :func:`mx8_quantize`, :func:`mx8_dequantize`: activations into an :class:`Mx8`
  (8.25 bits a value), which :func:`mx4_linear` takes for x, and back.
* :func:`rms_norm`: root-mean-square norms with a residual's addition, in x's type
  or in MX FP8.
* :func:`attention`: causal attention of packed sequences, with a sliding window and
  sinks; :func:`attention_cached`: the same of new tokens over a :class:`KvCache`.
* :func:`embedding`: scaled table rows by token, from a tensor or an
  :class:`Mx4`; :func:`embedding_grad`: the table's gradient.

Operators run on ``stream`` (by default the device's current stream) and return
without waiting.  Their outputs and workspaces belong to that stream; inputs
made on another one must be ready for it (``stream.wait_stream(...)``), and are
kept from reuse until it has passed the call.  ``mx4_linear``, ``embedding``,
``rms_norm`` and ``attention`` take part in autograd where one of their inputs
requires a gradient.  There is no forward mode: a tensor with a tangent is
refused.

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


class _Mx:
    """Codes and scales of a matrix in blocks of 32 columns."""

    __slots__ = ("_codes", "_scales", "_cols")
    _BLOCK_BYTES: int  # of codes

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int):
        self._codes, self._scales, self._cols = codes, scales, cols
        self._check()

    @classmethod
    def _pitches(cls, cols: int):
        blocks = -(-cols // BLOCK)
        return blocks * cls._BLOCK_BYTES, -(-blocks // 16) * 16

    def _check(self):
        cols = self._cols
        code_pitch, scale_pitch = self._pitches(cols)
        for name, t, pitch in (("codes", self._codes, code_pitch), ("scales", self._scales, scale_pitch)):
            if t.dtype != torch.uint8 or t.dim() != 2 or t.shape[1] != pitch or not t.is_contiguous():
                raise ValueError(f"{name}: expected a contiguous uint8 tensor of {pitch} columns for {cols} columns, "
                                 f"got {t.dtype} with shape {tuple(t.shape)} and strides {t.stride()}")
        if self._codes.shape[0] != self._scales.shape[0] or self._codes.device != self._scales.device:
            raise ValueError("codes and scales differ in rows or device")

    @classmethod
    def _of(cls, codes: torch.Tensor, scales: torch.Tensor, cols: int):
        """The same without a check."""
        q = cls.__new__(cls)
        q._codes, q._scales, q._cols = codes, scales, cols
        return q

    @classmethod
    def empty(cls, rows: int, cols: int, device):
        """A matrix whose contents are not set."""
        code_pitch, scale_pitch = cls._pitches(cols)
        return cls._of(torch.empty((rows, code_pitch), dtype=torch.uint8, device=device),
                       torch.empty((rows, scale_pitch), dtype=torch.uint8, device=device), cols)

    @classmethod
    def _beside(cls, t: torch.Tensor, rows: int, cols: int):
        """One whose contents are not set, where t is: half a microsecond less than by naming the device."""
        code_pitch, scale_pitch = cls._pitches(cols)
        return cls._of(t.new_empty((rows, code_pitch), dtype=torch.uint8), t.new_empty((rows, scale_pitch), dtype=torch.uint8), cols)

    def __reduce__(self):
        return type(self), (self._codes, self._scales, self._cols)

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

    def __getitem__(self, rows: slice):
        """A run of rows, sharing this matrix's memory."""
        if not isinstance(rows, slice) or rows.step not in (None, 1):
            raise ValueError(f"an {type(self).__name__} is indexed by a run of rows")
        return type(self)(self.codes[rows], self.scales[rows], self.cols)

    def __repr__(self):
        return f"{type(self).__name__}({self.rows} x {self.cols}, {self.device})"


class Mx4(_Mx):
    """A matrix in MX FP4: ``codes`` (rows, blocks * 16) and ``scales`` (rows,
    blocks rounded up to 16), both contiguous uint8, laid out as ``sllm_mx``.
    It is those tensors, wherever their storage is when it is used."""

    __slots__ = ()
    _BLOCK_BYTES = 16


class Mx8(_Mx):
    """Activations in MX FP8, 8.25 bits a value: as :class:`Mx4`, with ``codes`` (rows,
    blocks * 32), an E4M3 value each."""

    __slots__ = ()
    _BLOCK_BYTES = 32


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
    return (t._codes if isinstance(t, _Mx) else t).get_device()


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
            for u in ((t.codes, t.scales) if isinstance(t, _Mx) else (t,)):
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
    if not hasattr(ext, "attention_grad"):
        return None
    L = binding.lib()
    names = ("sllm_mx_quantize", "sllm_mx_dequantize", "sllm_mx_linear", "sllm_mx_linear_workspace", "sllm_mx_linear_mx",
             "sllm_mx_linear_mx_workspace", "sllm_mx_linear_grad", "sllm_mx_linear_grad_workspace", "sllm_embedding",
             "sllm_embedding_mx", "sllm_embedding_grad", "sllm_embedding_grad_workspace", "sllm_rms_norm", "sllm_rms_norm_octet",
             "sllm_rms_norm_grad", "sllm_rms_norm_grad_workspace", "sllm_mx_linear_octet", "sllm_mx_linear_octet_workspace",
             "sllm_attention", "sllm_attention_grad", "sllm_attention_grad_workspace", "sllm_attention_cached",
             "sllm_attention_cached_workspace")
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


def mx4_linear(x: Union[torch.Tensor, Mx4, Mx8], w: Mx4, out: Optional[torch.Tensor] = None,
               out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """``x @ w.T``: (..., w.rows) for x (..., w.cols).

    x as a tensor keeps its own precision; as an :class:`Mx4` both sides are in
    four bits, as an :class:`Mx8` x is in eight.  The result has ``out_dtype``, by
    default x's type (bfloat16 for an :class:`Mx4` or :class:`Mx8`)."""
    if stream is not None:
        return _on_stream(stream, mx4_linear, x, w, out, out_dtype, keep=(x, w, out))
    if isinstance(x, _Mx):
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
    if isinstance(x, Mx8):
        if out is None and device >= 0 and code is not None and _native() is not None:
            native = _native()
            y = native.ext.product_octet(native.mx_linear_octet, native.mx_linear_octet_workspace, x._codes, x._scales, x._cols, w._codes,
                                         w._scales, w._cols, code, device, _raw_stream(device))
            if y.__class__ is int:
                binding.check(y)
            if y is not None:
                return y
        L = binding.lib()
        y, rows = _output(out, (x.rows, w.rows), x.rows, w.rows, out_dtype or torch.bfloat16, x.codes)
        operands = x._struct, w._struct
        n = _workspace(L.sllm_mx_linear_octet_workspace, *operands, rows.dtype)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
        binding.check(L.sllm_mx_linear_octet(*operands, rows, ws.data_ptr() if n else None, n, device, _raw_stream(device)))
        _written(out)
        return y
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


def mx8_quantize(x: torch.Tensor, out: Optional[Mx8] = None, stream=None) -> Mx8:
    """The rows of x (its leading dimensions flattened) in MX FP8, for :func:`mx4_linear`.
    No gradient passes, as for :func:`mx4_quantize`."""
    if stream is not None:
        return _on_stream(stream, mx8_quantize, x, out, keep=(x, out))
    _refuse_tangent(x)
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError("x requires a gradient, which quantisation does not pass on")
    src = _matrix(x, "x")
    device = _one_device(x, out)
    q = Mx8._beside(x, src.rows, src.cols) if out is None else out
    if not isinstance(q, Mx8) or q.rows != src.rows or q.cols != src.cols:
        raise ValueError(f"out: expected an Mx8 of {src.rows} x {src.cols}, got {q!r}")
    binding.check(binding.lib().sllm_mx_octet_quantize(src, q._struct, device, _raw_stream(device)))
    if out is not None:
        _written(out.codes, out.scales)
    return q


def mx8_dequantize(q: Mx8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The values q stands for, rounded to ``dtype`` (or the type of ``out``)."""
    if stream is not None:
        return _on_stream(stream, mx8_dequantize, q, dtype, out, keep=(q, out))
    if not isinstance(q, Mx8):
        raise ValueError(f"expected an Mx8, got {q!r}")
    device = _index(q)
    y, rows = _output(out, (q.rows, q.cols), q.rows, q.cols, dtype, q.codes)
    binding.check(binding.lib().sllm_mx_octet_dequantize(q._struct, rows, device, _raw_stream(device)))
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


# ---------------------------------------------------------------------------
# norms
# ---------------------------------------------------------------------------

def _refuse_capture(x: torch.Tensor):
    # A captured backward pass that reaches a leaf which an eager graph holds too waits for
    # that leaf's stream, outside the capture, and ends the process.
    if x.is_cuda and torch.cuda.is_current_stream_capturing():
        raise ValueError("norms and attention pass no gradient under graph capture: capture them under torch.no_grad(), "
                         "or the entry points of their gradients")


def rms_norm(x: torch.Tensor, gain: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-5, mx8: bool = False,
             stream=None):
    """h / sqrt(mean h^2 + eps) * gain over the last dimension, in x's type, h being x, or
    with a residual ``x + residual`` rounded to their type: then the norm and h.

    ``gain`` may be of another type.  With ``mx8`` the norm is an :class:`Mx8`, its rows
    the leading dimensions flattened, and no gradient passes."""
    if stream is not None:
        return _on_stream(stream, rms_norm, x, gain, residual, eps, mx8, keep=(x, gain, residual))
    for t in (x, gain, residual):
        _refuse_tangent(t)
    if torch.is_grad_enabled() and (x.requires_grad or gain.requires_grad or (residual is not None and residual.requires_grad)):
        if mx8:
            raise ValueError("a tensor requires a gradient, which a norm in MX FP8 does not pass on")
        _refuse_capture(x)
        y, h = _RmsNorm.apply(x, gain, residual, eps)
        return y if residual is None else (y, h)
    device, native = x.get_device(), _native()
    if device >= 0 and native is not None:
        parts = native.ext.norm(native.rms_norm_octet if mx8 else native.rms_norm, x, gain, residual, eps, 1 if mx8 else 0, device,
                                _raw_stream(device))
        if parts.__class__ is int:
            binding.check(parts)
        if parts is not None:
            if not mx8:
                return parts
            y = Mx8._of(parts[0], parts[1], x.shape[-1])
            return y if residual is None else (y, parts[2])
    y, h, _ = _rms_norm(x, gain, residual, eps, mx8, False)
    return y if residual is None else (y, h)


def _rms_norm(x, gain, residual, eps, mx8, keep):
    """The norm, h and, with ``keep``, each row's inverse root mean square."""
    src, g = _matrix(x, "x"), _matrix(gain, "gain")
    if gain.dim() != 1:
        raise ValueError(f"gain: expected one dimension, got shape {tuple(gain.shape)}")
    device, r, h, rows = _one_device(x, gain, residual), None, x, None
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise ValueError(f"residual: expected {x.dtype} of shape {tuple(x.shape)}, got {residual.dtype} of shape {tuple(residual.shape)}")
        r = _matrix(residual, "residual")
        h, rows = _output(None, x.shape, src.rows, src.cols, x.dtype, x)
    L, stream = binding.lib(), _raw_stream(device)
    if mx8:
        y = Mx8._beside(x, src.rows, src.cols)
        binding.check(L.sllm_rms_norm_octet(src, r, g, eps, rows, y._struct, device, stream))
        return y, h, None
    y, y_rows = _output(None, x.shape, src.rows, src.cols, x.dtype, x)
    inverse = torch.empty(src.rows, dtype=torch.float32, device=x.device) if keep else None
    binding.check(L.sllm_rms_norm(src, r, g, eps, rows, y_rows, inverse.data_ptr() if keep else None, device, stream))
    return y, h, inverse


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, residual, eps):
        ctx.set_materialize_grads(False)
        parts, device, native = None, x.get_device(), _native()
        if device >= 0 and native is not None:
            parts = native.ext.norm_kept(native.rms_norm, x, gain, residual, eps, device, _raw_stream(device))
            if parts.__class__ is int:
                binding.check(parts)
        if parts is None:
            y, h, inverse = _rms_norm(x, gain, residual, eps, False, True)
        else:
            y, inverse, h = parts if residual is not None else (*parts, x)
        ctx.save_for_backward(h, gain, inverse)
        ctx.residual = residual is not None
        if residual is None:
            h = None
        return y, h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh):
        h, gain, inverse = ctx.saved_tensors
        if dy is None:  # h alone has been used
            return dh, None, dh if ctx.residual else None, None
        if not h.numel():
            dx = torch.zeros_like(h)
            return dx, torch.zeros_like(gain), dx if ctx.residual else None, None
        # gradients of sums and means arrive with strides of 0
        dy, dh, device, native = dy.contiguous(), None if dh is None else dh.contiguous(), h.get_device(), _native()
        if native is not None:
            parts = native.ext.norm_grad(native.rms_norm_grad, native.rms_norm_grad_workspace, dy, dh, h, gain, inverse, device,
                                         _raw_stream(device))
            if parts.__class__ is int:
                binding.check(parts)
            if parts is not None:
                return *parts, parts[0] if ctx.residual else None, None
        rows = _matrix(h, "h")
        dx, dx_rows = _output(None, h.shape, rows.rows, rows.cols, h.dtype, h)
        dgain = torch.empty(gain.shape, dtype=gain.dtype, device=gain.device)
        L = binding.lib()
        n = _workspace(L.sllm_rms_norm_grad_workspace, rows.rows, rows.cols)
        ws = torch.empty(n, dtype=torch.uint8, device=h.device) if n else None
        binding.check(L.sllm_rms_norm_grad(_matrix(dy, "dy"), None if dh is None else _matrix(dh, "dh"), rows, _matrix(gain, "gain"),
                                           inverse.data_ptr(), dx_rows, _matrix(dgain, "dgain"), ws.data_ptr() if n else None, n, device,
                                           _raw_stream(device)))
        return dx, dgain, dx if ctx.residual else None, None


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def _heads(t: torch.Tensor, name: str) -> binding.Heads:
    """(tokens, heads, elements) by their strides."""
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: {t.dtype} is not float32, float16 or bfloat16")
    if not t.is_cuda:
        raise ValueError(f"{name} is not in device memory")
    if t.is_neg():
        raise ValueError(f"{name} is a negated view of other elements")
    if t.dim() != 3:
        raise ValueError(f"{name}: expected tokens, heads and elements, got shape {tuple(t.shape)}")
    tokens, heads, dim = t.shape
    if not t.numel():
        return binding.Heads(t.data_ptr(), tokens, heads, dim, heads * dim, dim, code, 0)
    strides = t.stride()
    if dim > 1 and strides[2] != 1:
        raise ValueError(f"{name}: the elements of a head are not adjacent (strides {strides})")
    # a single token's or head's stride says nothing
    return binding.Heads(t.data_ptr(), tokens, heads, dim, strides[0] if tokens > 1 else heads * dim,
                         strides[1] if heads > 1 else dim, code, 0)


def _index_tensor(t: Optional[torch.Tensor], name: str) -> Optional[binding.Ids]:
    if t is None:
        return None
    if t.dim() != 1:
        raise ValueError(f"{name}: expected one dimension, got shape {tuple(t.shape)}")
    try:
        return _ids(t)
    except ValueError as e:
        raise ValueError(str(e).replace("tokens", name)) from None


class KvCache:
    """Keys and values of sequences, each (sequences, heads, sinks + window, elements) and
    contiguous: the first ``sinks`` positions of a sequence and the last ``window`` ones.
    Position p is in slot p, or from the sinks on in slot sinks + (p - sinks) % window.
    It is those tensors, wherever their storage is when it is used."""

    __slots__ = ("k", "v", "window", "sinks")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, window: int, sinks: int = 0):
        self.k, self.v, self.window, self.sinks = k, v, window, sinks
        self._check()

    def _check(self):
        if self.window < 1 or self.sinks < 0:
            raise ValueError(f"a window of {self.window} and {self.sinks} sinks")
        for name, t in (("k", self.k), ("v", self.v)):
            if t.dtype not in _DTYPE:
                raise ValueError(f"{name}: {t.dtype} is not float32, float16 or bfloat16")
            if t.dim() != 4 or t.shape[2] != self.sinks + self.window or not t.is_contiguous() or t.is_neg():
                raise ValueError(f"{name}: expected a contiguous tensor of sequences, heads, {self.sinks + self.window} slots and "
                                 f"elements, got shape {tuple(t.shape)} and strides {t.stride()}")
        if self.k.shape != self.v.shape or self.k.dtype != self.v.dtype or self.k.device != self.v.device:
            raise ValueError("k and v differ in shape, type or device")

    @classmethod
    def empty(cls, sequences: int, heads: int, dim: int, window: int, sinks: int = 0, dtype=torch.bfloat16, device=None) -> "KvCache":
        """A cache whose contents are not set, for sequences that have had no tokens."""
        shape = (sequences, heads, sinks + window, dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device), window, sinks)

    @property
    def _struct(self) -> binding.KvCache:
        self._check()
        n, heads, _, dim = self.k.shape
        return binding.KvCache(self.k.data_ptr(), self.v.data_ptr(), n, heads, dim, self.window, self.sinks, _DTYPE[self.k.dtype], 0)

    @property
    def device(self):
        return self.k.device

    def __getitem__(self, sequences: slice) -> "KvCache":
        """A run of sequences, sharing this cache's memory."""
        if not isinstance(sequences, slice) or sequences.step not in (None, 1):
            raise ValueError("a KvCache is indexed by a run of sequences")
        return KvCache(self.k[sequences], self.v[sequences], self.window, self.sinks)

    def __repr__(self):
        n, heads, _, dim = self.k.shape
        return f"KvCache({n} x {heads} x ({self.sinks} + {self.window}) x {dim}, {self.k.dtype}, {self.device})"


def _out_heads(out: Optional[torch.Tensor], like: torch.Tensor):
    if out is None:
        out = like.new_empty(like.shape)
    elif out.shape != like.shape or out.dtype != like.dtype or out.device != like.device:
        raise ValueError(f"out: expected {like.dtype} of shape {tuple(like.shape)} on {like.device}, "
                         f"got {out.dtype} of shape {tuple(out.shape)} on {out.device}")
    else:
        _refuse_tangent(out)
        _refuse_grad(out)
    return out, _heads(out, "out")


def _window(window: Optional[int], sinks: int) -> int:
    if (window is not None and window < 1) or sinks < 0:
        raise ValueError(f"a window of {window} and {sinks} sinks")
    return min(window or 0, 1 << 62)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, window: Optional[int] = None, sinks: int = 0,
              offsets: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """Causal attention of packed sequences: (tokens, heads, elements) for q of that shape
    and k and v of (tokens, key/value heads, elements), heads a multiple of theirs.

    The query at position i of its sequence sees the key at position j of the same one
    where j <= i and (i - j < window or j < sinks); without a window every j <= i.
    ``offsets`` (int32 or int64, one more than there are sequences) tells where each
    starts and the last one ends; without it all tokens are one sequence.  Tokens of no
    sequence are padding: rows of zeros, whose gradients are zeros.  ``scale`` is
    elements ** -0.5 if not given."""
    if stream is not None:
        return _on_stream(stream, attention, q, k, v, window, sinks, offsets, scale, out, keep=(q, k, v, offsets, out))
    for t in (q, k, v):
        _refuse_tangent(t)
    if scale is None:
        scale = q.shape[-1] ** -0.5 if q.dim() and q.shape[-1] else 1.0
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        if out is not None:
            raise ValueError("an operator that writes to a given tensor takes no part in autograd")
        _refuse_capture(q)
        return _Attention.apply(q, k, v, window, sinks, offsets, scale)
    device, native = q.get_device(), _native()
    if out is None and device >= 0 and native is not None:
        y = native.ext.attention(native.attention, q, k, v, offsets, _window(window, sinks), min(sinks, 1 << 62), scale, device, _raw_stream(device), 0)
        if y.__class__ is int:
            binding.check(y)
        if y is not None:
            return y
    return _attention(q, k, v, window, sinks, offsets, scale, out, None)


def _attention(q, k, v, window, sinks, offsets, scale, out, lse):
    window, args, ids = _window(window, sinks), (_heads(q, "q"), _heads(k, "k"), _heads(v, "v")), _index_tensor(offsets, "offsets")
    device = _one_device(q, k, v, offsets)
    y, rows = _out_heads(out, q)
    binding.check(binding.lib().sllm_attention(*args, ids, window, min(sinks, 1 << 62), scale, rows,
                                               None if lse is None else lse.data_ptr(), device, _raw_stream(device)))
    _written(out)
    return y


def attention_cached(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cache: KvCache, lengths: torch.Tensor,
                     offsets: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """:func:`attention` of new tokens behind those that ``cache`` holds, with its window
    and sinks; their keys and values are written into it.

    ``lengths`` (int32 or int64) is how many tokens each sequence has had before, and where
    its new ones start; it is only read.  The new tokens of a sequence are those between
    its ``offsets``, or without them one for each sequence, in their order.  A sequence
    whose length is negative takes no part: its rows are zeros, its cache stays.  No
    gradient passes."""
    if stream is not None:
        return _on_stream(stream, attention_cached, q, k, v, cache, lengths, offsets, scale, out,
                          keep=(q, k, v, cache.k, cache.v, lengths, offsets, out))
    for t in (q, k, v, cache.k, cache.v):
        _refuse_tangent(t)
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError("a tensor requires a gradient, which attention over a cache does not pass on")
    if scale is None:
        scale = q.shape[-1] ** -0.5 if q.dim() and q.shape[-1] else 1.0
    if lengths is None:
        raise ValueError("lengths: None")
    device, native = q.get_device(), _native()
    if out is None and device >= 0 and native is not None:
        y = native.ext.attention_cached(native.attention_cached, native.attention_cached_workspace, q, k, v, cache.k, cache.v, cache.window,
                                        cache.sinks, lengths, offsets, scale, device, _raw_stream(device))
        if y.__class__ is int:
            binding.check(y)
        if y is not None:
            _written(None, cache.k, cache.v)
            return y
    args = (_heads(q, "q"), _heads(k, "k"), _heads(v, "v"), cache._struct, _index_tensor(lengths, "lengths"), _index_tensor(offsets, "offsets"))
    device = _one_device(q, k, v, cache.k, lengths, offsets)
    y, rows = _out_heads(out, q)
    L = binding.lib()
    n = _workspace(L.sllm_attention_cached_workspace, *args)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    binding.check(L.sllm_attention_cached(*args, scale, rows, ws.data_ptr() if n else None, n, device, _raw_stream(device)))
    _written(out, cache.k, cache.v)
    return y


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, sinks, offsets, scale):
        parts, device, native = None, q.get_device(), _native()
        if device >= 0 and native is not None:
            parts = native.ext.attention(native.attention, q, k, v, offsets, _window(window, sinks), min(sinks, 1 << 62), scale, device,
                                         _raw_stream(device), 1)
            if parts.__class__ is int:
                binding.check(parts)
        if parts is None:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
            out = _attention(q, k, v, window, sinks, offsets, scale, None, lse)
        else:
            out, lse = parts
        ctx.save_for_backward(q, k, v, out, lse, offsets)
        ctx.window, ctx.sinks, ctx.scale = window, sinks, scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, offsets = ctx.saved_tensors
        dout = dout.contiguous()  # gradients of sums and means arrive with strides of 0
        device, native = q.get_device(), _native()
        if native is not None:
            parts = native.ext.attention_grad(native.attention_grad, native.attention_grad_workspace, dout, q, k, v, out, lse, offsets,
                                              _window(ctx.window, ctx.sinks), min(ctx.sinks, 1 << 62), ctx.scale, device, _raw_stream(device))
            if parts.__class__ is int:
                binding.check(parts)
            if parts is not None:
                return *parts, None, None, None, None
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        L, ids = binding.lib(), _index_tensor(offsets, "offsets")
        rows = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
        window, sinks = _window(ctx.window, ctx.sinks), min(ctx.sinks, 1 << 62)
        n = _workspace(L.sllm_attention_grad_workspace, *rows[:2], ids, window, sinks)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
        binding.check(L.sllm_attention_grad(
            _heads(dout, "dout"), *rows, _heads(out, "out"), lse.data_ptr(), ids, window, sinks,
            ctx.scale, _heads(dq, "dq"), _heads(dk, "dk"), _heads(dv, "dv"), ws.data_ptr() if n else None, n, device, _raw_stream(device)))
        return dq, dk, dv, None, None, None, None
