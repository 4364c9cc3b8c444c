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
take part in autograd where their input or table requires a gradient.

Rows may be apart by any stride, but the elements of a row must be adjacent:
other tensors are refused, not copied.
"""

from __future__ import annotations

import ctypes as C
from typing import Optional, Union

import torch

from paper_2401_14351_amd import binding

BLOCK = 32  # columns that share a scale

_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_ID_BITS = {torch.int32: 32, torch.int64: 64}


def _pitches(cols: int):
    blocks = -(-cols // BLOCK)
    return blocks * 16, -(-blocks // 16) * 16


class Mx4:
    """A matrix in MX FP4: ``codes`` (rows, blocks * 16) and ``scales`` (rows,
    blocks rounded up to 16), both contiguous uint8, laid out as ``sllm_mx``."""

    __slots__ = ("codes", "scales", "rows", "cols", "_struct")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int):
        code_pitch, scale_pitch = _pitches(cols)
        for name, t, pitch in (("codes", codes, code_pitch), ("scales", scales, scale_pitch)):
            if t.dtype != torch.uint8 or t.dim() != 2 or t.shape[1] != pitch or not t.is_contiguous():
                raise ValueError(f"{name}: expected a contiguous uint8 tensor of {pitch} columns for {cols} columns, "
                                 f"got {t.dtype} with shape {tuple(t.shape)} and strides {t.stride()}")
        if codes.shape[0] != scales.shape[0] or codes.device != scales.device:
            raise ValueError("codes and scales differ in rows or device")
        self.codes, self.scales = codes, scales
        self.rows, self.cols = codes.shape[0], cols
        self._struct = binding.Mx(codes.data_ptr(), scales.data_ptr(), self.rows, cols)

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Mx4":
        """A matrix whose contents are not set."""
        code_pitch, scale_pitch = _pitches(cols)
        return cls(torch.empty(rows, code_pitch, dtype=torch.uint8, device=device),
                   torch.empty(rows, scale_pitch, dtype=torch.uint8, device=device), cols)

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
    if t.dim() == 0:
        raise ValueError(f"{name} has no dimensions")
    cols = t.shape[-1]
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row are not adjacent (strides {t.stride()})")
    if t.dim() == 1:
        return binding.Matrix(t.data_ptr(), 1, cols, cols, code, 0)
    if t.dim() > 2:
        rows = t.numel() // cols if cols else t.shape[:-1].numel()
        if rows and cols:
            try:
                t = t.view(rows, cols)
            except RuntimeError:
                raise ValueError(f"{name}: its rows are not apart by one stride (strides {t.stride()})") from None
        else:
            return binding.Matrix(t.data_ptr(), rows, cols, cols, code, 0)
    # a single row's or no row's stride says nothing
    return binding.Matrix(t.data_ptr(), t.shape[0], cols, t.stride(0) if t.shape[0] > 1 else cols, code, 0)


def _ids(t: torch.Tensor) -> binding.Ids:
    bits = _ID_BITS.get(t.dtype)
    if bits is None:
        raise ValueError(f"tokens: {t.dtype} is not int32 or int64")
    if not t.is_cuda:
        raise ValueError("tokens are not in device memory")
    if not t.is_contiguous():
        raise ValueError(f"tokens are not contiguous (strides {t.stride()})")
    return binding.Ids(t.data_ptr(), t.numel(), bits, 0)


class _On:
    """The stream of a call: what is allocated inside belongs to it, and its
    inputs are kept from reuse until it has passed the call."""

    __slots__ = ("device", "ptr", "_stream", "_context")

    def __init__(self, device: torch.device, stream, *inputs):
        for t in inputs:
            if t.device != device:
                raise ValueError(f"inputs on {device} and {t.device}")
        self.device = device.index
        self._context = None
        if stream is None:
            self.ptr = torch.cuda.current_stream(device).cuda_stream
            return
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream, device=device)
        self.ptr = stream.cuda_stream
        self._context = torch.cuda.stream(stream)
        for t in inputs:
            for u in ((t.codes, t.scales) if isinstance(t, Mx4) else (t,)):
                u.record_stream(stream)

    def __enter__(self):
        if self._context is not None:
            self._context.__enter__()
        return self

    def __exit__(self, *exc):
        if self._context is not None:
            self._context.__exit__(*exc)


def _output(out: Optional[torch.Tensor], shape, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if out.shape != torch.Size(shape) or out.device != device:
        raise ValueError(f"out: expected shape {tuple(shape)} on {device}, got {tuple(out.shape)} on {out.device}")
    return out


def _refuse_grad(*tensors):
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("an operator that writes to a given tensor takes no part in autograd")


def mx4_quantize(x: torch.Tensor, out: Optional[Mx4] = None, stream=None) -> Mx4:
    """The rows of x (its leading dimensions flattened) in MX FP4."""
    src = _matrix(x, "x")
    if out is not None and out.shape != (src.rows, src.cols):
        raise ValueError(f"out: expected {src.rows} x {src.cols}, got {out.rows} x {out.cols}")
    with _On(x.device, stream, x, *(() if out is None else (out,))) as on:
        if out is None:
            out = Mx4.empty(src.rows, src.cols, x.device)
        binding.check(binding.lib().sllm_mx_quantize(src, out._struct, on.device, on.ptr))
    return out


def mx4_dequantize(q: Mx4, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The values q stands for, rounded to ``dtype`` (or the type of ``out``)."""
    _refuse_grad(out)
    with _On(q.device, stream, q, *(() if out is None else (out,))) as on:
        out = _output(out, (q.rows, q.cols), dtype, q.device)
        binding.check(binding.lib().sllm_mx_dequantize(q._struct, _matrix(out, "out"), on.device, on.ptr))
    return out


def _workspace(query, *args) -> int:
    """How many bytes of workspace a call with these operands needs."""
    n = C.c_uint64()
    binding.check(query(*args, n))
    return n.value


def mx4_linear(x: Union[torch.Tensor, Mx4], w: Mx4, out: Optional[torch.Tensor] = None,
               out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """``x @ w.T``: (..., w.rows) for x (..., w.cols).

    x as a tensor keeps its own precision; as an :class:`Mx4` both sides are in
    four bits.  The result has ``out_dtype``, by default x's type (bfloat16 for
    an :class:`Mx4`)."""
    if isinstance(x, Mx4):
        _refuse_grad(out)
        return _linear_mx(x, w, out, out_dtype, stream)
    if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
        _refuse_grad(out)
        if out is not None:
            raise ValueError("an operator that writes to a given tensor takes no part in autograd")
        return _Linear.apply(x, w, out_dtype, stream)
    return _linear(x, w, out, out_dtype, stream)


def _linear(x, w, out, out_dtype, stream):
    L = binding.lib()
    xs = _matrix(x, "x")
    with _On(x.device, stream, x, w, *(() if out is None else (out,))) as on:
        out = _output(out, x.shape[:-1] + (w.rows,), out_dtype or x.dtype, x.device)
        n = _workspace(L.sllm_mx_linear_workspace, xs, w._struct)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
        binding.check(L.sllm_mx_linear(xs, w._struct, _matrix(out, "out"), ws.data_ptr() if n else None, n, on.device,
                                       on.ptr))
    return out


def _linear_mx(x, w, out, out_dtype, stream):
    L = binding.lib()
    with _On(x.device, stream, x, w, *(() if out is None else (out,))) as on:
        out = _output(out, (x.rows, w.rows), out_dtype or torch.bfloat16, x.device)
        n = _workspace(L.sllm_mx_linear_mx_workspace, x._struct, w._struct)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
        binding.check(L.sllm_mx_linear_mx(x._struct, w._struct, _matrix(out, "out"), ws.data_ptr() if n else None, n,
                                          on.device, on.ptr))
    return out


def mx4_linear_grad(dy: torch.Tensor, w: Mx4, out: Optional[torch.Tensor] = None,
                    out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """``dy @ w``, the gradient of :func:`mx4_linear` by x: (..., w.cols) for dy
    (..., w.rows)."""
    _refuse_grad(dy, out)
    L = binding.lib()
    ds = _matrix(dy, "dy")
    with _On(dy.device, stream, dy, w, *(() if out is None else (out,))) as on:
        out = _output(out, dy.shape[:-1] + (w.cols,), out_dtype or dy.dtype, dy.device)
        n = _workspace(L.sllm_mx_linear_grad_workspace, ds, w._struct)
        ws = torch.empty(n, dtype=torch.uint8, device=dy.device) if n else None
        binding.check(L.sllm_mx_linear_grad(ds, w._struct, _matrix(out, "out"), ws.data_ptr() if n else None, n,
                                            on.device, on.ptr))
    return out


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, out_dtype, stream):
        ctx.w, ctx.dtype = w, x.dtype
        return _linear(x, w, None, out_dtype, stream)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        # gradients of sums and means arrive with strides of 0
        return mx4_linear_grad(dy.contiguous(), ctx.w, out_dtype=ctx.dtype), None, None, None


def embedding(table: Union[torch.Tensor, Mx4], tokens: torch.Tensor, scale: float = 1.0,
              out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
              stream=None) -> torch.Tensor:
    """``scale`` times the table's rows of ``tokens`` (int32 or int64): shape
    ``tokens.shape + (columns,)``, in ``out_dtype`` (by default the table's
    type, bfloat16 for an :class:`Mx4`).  A token outside the table is padding:
    a row of zeros."""
    if not isinstance(table, Mx4) and torch.is_grad_enabled() and table.requires_grad:
        _refuse_grad(out)
        if out is not None:
            raise ValueError("an operator that writes to a given tensor takes no part in autograd")
        return _Embedding.apply(table, tokens, scale, out_dtype, stream)
    return _embedding(table, tokens, scale, out, out_dtype, stream)


def _embedding(table, tokens, scale, out, out_dtype, stream):
    L = binding.lib()
    ids = _ids(tokens)
    mx = isinstance(table, Mx4)
    if not mx and table.dim() != 2:
        raise ValueError(f"table: expected rows and columns, got shape {tuple(table.shape)}")
    with _On(table.device, stream, table, tokens, *(() if out is None else (out,))) as on:
        cols = table.cols if mx else table.shape[1]
        out = _output(out, tokens.shape + (cols,), out_dtype or (torch.bfloat16 if mx else table.dtype), table.device)
        fn = L.sllm_embedding_mx if mx else L.sllm_embedding
        binding.check(fn(table._struct if mx else _matrix(table, "table"), ids, scale, _matrix(out, "out"), on.device,
                         on.ptr))
    return out


def embedding_grad(dy: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0,
                   out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                   accumulate: bool = False, stream=None) -> torch.Tensor:
    """The gradient of :func:`embedding` by a table of ``vocab`` rows: row v is
    ``scale`` times the sum of dy over the positions of token v, in their order.
    ``accumulate`` adds it to ``out`` instead of replacing its contents."""
    _refuse_grad(dy, out)
    if accumulate and out is None:
        raise ValueError("accumulate needs a gradient to add to")
    if dy.shape[:-1] != tokens.shape:
        raise ValueError(f"dy of shape {tuple(dy.shape)} for tokens of shape {tuple(tokens.shape)}")
    L = binding.lib()
    ids, ds = _ids(tokens), _matrix(dy, "dy")
    with _On(dy.device, stream, dy, tokens, *(() if out is None else (out,))) as on:
        out = _output(out, (vocab, dy.shape[-1]), out_dtype or dy.dtype, dy.device)
        grad = _matrix(out, "out")
        n = _workspace(L.sllm_embedding_grad_workspace, ids.n, grad)
        ws = torch.empty(n, dtype=torch.uint8, device=dy.device) if n else None
        binding.check(L.sllm_embedding_grad(ds, ids, scale, 1 if accumulate else 0, grad, ws.data_ptr() if n else None, n,
                                            on.device, on.ptr))
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, out_dtype, stream):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.dtype, ctx.scale = table.shape[0], table.dtype, scale
        return _embedding(table, tokens, scale, None, out_dtype, stream)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        (tokens,) = ctx.saved_tensors
        return embedding_grad(dy.contiguous(), tokens, ctx.vocab, ctx.scale, out_dtype=ctx.dtype), None, None, None, None
