"""Embeddings of token ids with scaling, and their gradient by sorted ids: where a policy over token ids begins.

    x = embedding(table, tokens, scale=D ** 0.5, lengths=lengths)       # differentiable in the table
    g = embedding_grad(d_x, tokens, V, scale=D ** 0.5, lengths=lengths)  # the gradient alone
    embedding_grad(d_x, tokens, V, out=head_grad, accumulate=True)       # of a table that is the head's, too

Common arguments
  tokens       [B, T] or [N] (packed positions), int32 or int64
  lengths      [B]: position t of sequence b counts if t < lengths[b].  Not for packed positions
  mask         bool or uint8, of the tokens' shape: a position counts if it is not 0
  scale        of the embeddings
  status       int32 [1] on the GPU; TB_DEV_TOKEN_RANGE / TB_DEV_LENGTH_RANGE are OR-ed into it

What stands at positions that do not count has no part in anything; their embeddings are 0.  A table's gradient is
summed in float32 in an order that does not change from call to call.  Gradients are for reverse mode, and of first
order; tables with a forward-mode tangent are refused, and so is a backward pass that is captured into a HIP graph
while a graph from outside the capture, on the default stream, holds the table or the leaf that it comes from.
Everything runs on the current stream of the table's (or rows') GPU, and nothing synchronises.  See
include/tensorembed.h.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding as _b
from .binding import TensorBLEUError
from .losses import TYPES, _stay_in_capture, tb_positions_t

WIDTH_MOST = 1 << 20

EXPORTS = ["tensorembed_gradient", "tensorembed_lookup", "tensorembed_workspace_bytes"]

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class tb_table_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("row_stride", _i64), ("V", _i32), ("D", _i32), ("type", _i32)]


class tb_embedding_rows_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("seq_stride", _i64), ("pos_stride", _i64), ("B", _i32), ("T", _i32), ("D", _i32),
                ("type", _i32)]


class tb_table_gradient_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("row_stride", _i64), ("V", _i32), ("type", _i32), ("scale", _f32), ("accumulate", _i32)]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib = _b.load_library()
        p = ctypes.POINTER
        lib.tensorembed_lookup.restype = lib.tensorembed_gradient.restype = ctypes.c_int
        lib.tensorembed_lookup.argtypes = [p(tb_table_t), p(tb_positions_t), _i32, _i32, _f32, _vp, _vp, _vp]
        lib.tensorembed_gradient.argtypes = [p(tb_embedding_rows_t), p(tb_positions_t), p(tb_table_gradient_t), _vp, _vp,
                                             ctypes.c_size_t, _vp]
        lib.tensorembed_workspace_bytes.restype = ctypes.c_size_t
        lib.tensorembed_workspace_bytes.argtypes = [_i32] * 4
        _lib = lib
    return _lib


_host = None


def native():
    """The native marshalling module (built with the library; raises if it has not been).  Its functions
    return None for what they leave to the code here."""
    global _host
    if _host is None:
        _library()
        try:
            from . import _embed_host as module
        except ImportError as e:
            raise TensorBLEUError("the module _embed_host does not load: run `python -m "
                                  f"paper_2510_05485_amd.build` first ({e})") from e
        _host = module
    return _host


def workspace_bytes(B: int, T: int, V: int, D: int) -> int:
    return int(_library().tensorembed_workspace_bytes(B, T, V, D))


def _on(t, device, name: str) -> None:
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise TensorBLEUError(f"{name} must be a tensor on the GPU of the call "
                              f"(got {getattr(t, 'device', type(t).__name__)})")


def _values(t, dims, name):
    """A tensor of values on the GPU, detached, its rows' values next to one another."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TensorBLEUError(f"{name} must live on the GPU (got {getattr(t, 'device', type(t).__name__)})")
    if t.dtype not in TYPES:
        raise TensorBLEUError(f"{name} must be float32, bfloat16 or float16 (got {t.dtype})")
    if t.dim() not in dims or not 1 <= t.shape[-1] <= WIDTH_MOST:
        raise TensorBLEUError(f"{name}: unexpected shape {tuple(t.shape)}")
    if torch.autograd.forward_ad.unpack_dual(t).tangent is not None:
        raise TensorBLEUError(f"embeddings have no forward-mode derivative ({name} carries a tangent)")
    t = t.detach()
    return t if t.shape[-1] == 1 or t.stride(-1) == 1 else t.contiguous()


class _Positions:
    """Checked tokens, lengths, mask and status as the C struct; keeps what was converted alive."""

    def __init__(self, tokens, lengths, mask, status, device):
        _on(tokens, device, "tokens")
        if tokens.dtype not in (torch.int32, torch.int64) or tokens.dim() not in (1, 2):
            raise TensorBLEUError(f"tokens must be int32 or int64 of shape [B, T] or [N] (got {tokens.dtype} {tuple(tokens.shape)})")
        self.shape, self.device, self.keep = tuple(tokens.shape), device, []
        packed = tokens.dim() == 1
        self.B, self.T = (1, *self.shape) if packed else self.shape
        if self.B * self.T >= 2 ** 31 - 1:
            raise TensorBLEUError("too many positions for 32-bit counts")
        at = tb_positions_t()
        if self.T > 1 and tokens.stride(-1) != 1:
            tokens = tokens.contiguous()
        at.tokens, at.token_bytes = self._kept(tokens).data_ptr(), tokens.element_size()
        at.token_stride = self.T if packed else tokens.stride(0)
        if lengths is not None:
            if packed:
                raise TensorBLEUError("lengths are for tokens [B, T]; packed positions take a mask")
            _on(lengths, device, "lengths")
            if lengths.dtype not in (torch.int32, torch.int64) or tuple(lengths.shape) != (self.B,):
                raise TensorBLEUError(f"lengths must be int32 or int64 of shape {(self.B,)} "
                                      f"(got {lengths.dtype} {tuple(lengths.shape)})")
            if lengths.dtype == torch.int64:       # (wrong ones stay wrong when they are narrowed)
                lengths = lengths.clamp(-1, self.T + 1).to(torch.int32)
            at.lengths = self._kept(lengths.contiguous()).data_ptr()
        if mask is not None:
            _on(mask, device, "mask")
            if mask.dtype not in (torch.bool, torch.uint8) or tuple(mask.shape) != self.shape:
                raise TensorBLEUError(f"mask must be bool or uint8 of shape {self.shape} "
                                      f"(got {mask.dtype} {tuple(mask.shape)})")
            at.mask = self._kept(mask.contiguous()).data_ptr()
        if status is not None:
            _on(status, device, "status")
            if status.dtype != torch.int32 or status.numel() != 1:
                raise TensorBLEUError("status must be an int32 tensor of one element")
        self.at, self.status = at, None if status is None else status.data_ptr()

    def _kept(self, t):
        self.keep.append(t)
        return t


def _stream(device) -> int:
    return int(torch.cuda.current_stream(device).cuda_stream)


def _lookup(table, tokens, lengths, mask, scale, status):
    table = _values(table, (2,), "the table [V, D]")
    if not 1 <= table.shape[0] < 2 ** 31:
        raise TensorBLEUError(f"the table [V, D]: unexpected shape {tuple(table.shape)}")
    p = _Positions(tokens, lengths, mask, status, table.device)
    t = tb_table_t(table.data_ptr(), table.stride(0), *table.shape, TYPES[table.dtype])
    out = torch.empty(*p.shape, table.shape[1], dtype=table.dtype, device=table.device)
    with torch.cuda.device(table.device):
        rc = _library().tensorembed_lookup(ctypes.byref(t), ctypes.byref(p.at), p.B, p.T, float(scale), out.data_ptr(),
                                           p.status, _stream(table.device))
    _b._check(rc, "tensorembed_lookup")
    return out


def _gradient(rows, tokens, V, lengths, mask, scale, out, accumulate, status):
    p = _Positions(tokens, lengths, mask, status, rows.device)
    D = rows.shape[-1]
    if tuple(rows.shape[:-1]) != p.shape:
        raise TensorBLEUError(f"rows must be of shape {(*p.shape, 'D')} (got {tuple(rows.shape)})")
    strides = (0, rows.stride(0)) if rows.dim() == 2 else rows.stride()[:2]
    r = tb_embedding_rows_t(rows.data_ptr(), *strides, p.B, p.T, D, TYPES[rows.dtype])
    g = tb_table_gradient_t(out.data_ptr(), out.stride(0), V, TYPES[out.dtype], float(scale), int(accumulate))
    with torch.cuda.device(rows.device):
        n = workspace_bytes(p.B, p.T, V, D)
        w = torch.empty(n, dtype=torch.uint8, device=rows.device)
        rc = _library().tensorembed_gradient(ctypes.byref(r), ctypes.byref(p.at), ctypes.byref(g), p.status, w.data_ptr(), n,
                                             _stream(rows.device))
    _b._check(rc, "tensorembed_gradient")
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, lengths, mask, scale, status):
        out = _lookup(table, tokens, lengths, mask, scale, status)
        ctx.save_for_backward(tokens, lengths, mask)
        ctx.table, ctx.scale = (tuple(table.shape), table.dtype), scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_rows):
        _stay_in_capture()
        tokens, lengths, mask = ctx.saved_tensors
        (V, D), dtype = ctx.table
        rows = _values(d_rows.to(dtype), (2, 3), "the embeddings' gradient")
        out = torch.empty(V, D, dtype=dtype, device=rows.device)
        return (_gradient(rows, tokens, V, lengths, mask, ctx.scale, out, False, None), *(None,) * 5)


def embedding(table, tokens, *, scale: float = 1.0, lengths=None, mask=None,
              status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale times the rows of `table` [V, D] that `tokens` name: [B, T, D] or [N, D], of the table's type, rounded
    once.  Differentiable in the table.  A token outside the table has an embedding of NaN and no part in the
    gradient."""
    out = native().lookup(table, tokens, lengths, mask, scale, status)
    if out is not None:
        return out
    if isinstance(table, torch.Tensor) and torch.is_grad_enabled() and table.requires_grad:
        _values(table, (2,), "the table [V, D]")           # (a tangent is not to be seen inside a Function's forward)
        return _Embedding.apply(table, tokens, lengths, mask, scale, status)
    return _lookup(table, tokens, lengths, mask, scale, status)


def embedding_grad(rows, tokens, V: int, *, scale: float = 1.0, lengths=None, mask=None,
                   dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, accumulate: bool = False,
                   status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient [V, D] of embedding(...) in its table, from `rows`, that of the embeddings.

    dtype: the rows' (default) or float32.  out: where it goes (default: a new tensor); every row of it is
    written, or with `accumulate` those of tokens that come up are added to and no other one is touched (gradient
    accumulation; a table that has a gradient from elsewhere already)."""
    kind = isinstance(rows, torch.Tensor) and (dtype or (rows.dtype if out is None else getattr(out, "dtype", None)))
    wide = 1 if kind is torch.float32 else 0
    found = native().gradient(rows, tokens, V, lengths, mask, scale, wide, out, accumulate, status) \
        if wide or (isinstance(rows, torch.Tensor) and kind is rows.dtype) else None
    if found is not None:
        return found
    rows = _values(rows, (2, 3), "rows [B, T, D] or [N, D]")
    if isinstance(V, bool) or not isinstance(V, int) or not 1 <= V < 2 ** 31:
        raise TensorBLEUError(f"V must be a number of rows (got {V!r})")
    if kind not in (rows.dtype, torch.float32):
        raise TensorBLEUError(f"dtype must be {rows.dtype} or float32 (got {kind})")
    shape = (V, rows.shape[-1])
    if out is None:
        if accumulate:
            raise TensorBLEUError("accumulate needs out")
        return _gradient(rows, tokens, V, lengths, mask, scale, torch.empty(shape, dtype=kind, device=rows.device), False, status)
    _on(out, rows.device, "out")
    if out.dtype != kind or tuple(out.shape) != shape or (shape[1] > 1 and out.stride(-1) != 1):
        raise TensorBLEUError(f"out must be {kind} of shape {shape} with consecutive values in a row "
                              f"(got {out.dtype} {tuple(out.shape)})")
    if out.requires_grad and torch.is_grad_enabled():
        raise TensorBLEUError("out must not require a gradient")
    _gradient(rows, tokens, V, lengths, mask, scale, out.detach(), bool(accumulate), status)
    if not out.is_inference():
        torch.autograd.graph.increment_version(out)
    return out
