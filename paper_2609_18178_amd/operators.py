"""Training operators: block-scaled FP8 linear layers and the distillation loss.

What turns the BF16 working copy that a commit writes into the gradient that the
next commit reads.  The calls are thin: they check their tensors, allocate
outputs and scratch that the caller does not bring (torch's caching allocator,
on the current stream) and enqueue the library's kernels on torch's current HIP
stream; every computation runs in those kernels.  The mathematics, layouts and
edge cases are stated in ``include/pactshard.h``.

A training step of one linear layer::

    w = fp8_quantize(weight, square=True)                        # once after a commit
    w_t = fp8_quantize(weight, "columns", square=True)
    rows, columns = fp8_quantize(x, "both")                      # forward, x kept for the backward pass
    y = fp8_matmul(rows, w)
    ...
    dx, dw = fp8_linear_backward(dy, w_t, columns, grad_weight=grad, accumulate=True)

The calls are outside of autograd: a result has no graph, whatever its inputs require, and
gradients are what ``fp8_linear_backward`` and ``distill_grad`` or ``distill_step`` return
(an ``autograd.Function`` can be made of them). What is written into a tensor that a caller
hands over (``out``, ``grad``, ``grad_weight``) counts for autograd as changed in place.

A small call's time is the host's: what is below reads each property of a tensor
once and allocates once for what lives and dies together.
"""
from __future__ import annotations

import functools
import struct
from typing import Optional, Tuple, Union

import torch

from . import PACT_EINVAL, PACT_OK, PactError, _lib

__all__ = [
    "Fp8Matrix", "fp8_quantize", "fp8_matmul", "fp8_linear", "fp8_linear_backward",
    "distill_loss", "distill_grad", "distill_step",
]

FP8_BLOCK = 128
DISTILL_MAX_TOP = 1024
_FLAG_SQUARE = 1
_FLAG_ACCUMULATE = 1

# pact_matrix, pact_fp8 and pact_distill as bytes: packing is a fraction of what filling
# ctypes structures costs, and these calls start at a few microseconds
_MATRIX = struct.Struct("@4Q2I")
_FP8 = struct.Struct("@6Q")
_DISTILL = struct.Struct("@14Qf4I4xQ")
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_BYTES = {torch.uint8: 0}
_INDEX = {torch.int32: 4, torch.int64: 8}

_Tensor = torch.Tensor
_empty = torch.empty
_changed = torch._C._increment_version  # (torch.autograd.graph.increment_version at a third of its time)
_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream


def _pad(n: int, to: int) -> int:
    return (n + to - 1) // to * to


def _refuse(t, name: str, dtypes, index) -> None:
    """Says what is wrong with a tensor that is not a matrix of one of `dtypes` on GPU `index`."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise TypeError(f"{name} must live on a GPU (got {t.device}); there is no CPU path")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be one of {[str(d) for d in dtypes]}, not {t.dtype}")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{index}: one call runs on one GPU")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, not {t.dim()}")
    raise ValueError(f"the elements of a row of {name} must be neighbours and its rows apart (strides {tuple(t.stride())})")


def _matrix(t, name: str, index=None, dtypes=_DTYPES) -> Tuple[int, int, int, int]:
    """(rows, cols, elements between rows, element type) of a matrix on GPU `index` whose rows are contiguous."""
    if not isinstance(t, _Tensor) or not t.is_cuda or (index is not None and t.get_device() != index) or t.dim() != 2:
        _refuse(t, name, dtypes, index)
    kind = dtypes.get(t.dtype)
    if kind is None:
        _refuse(t, name, dtypes, index)
    rows, cols = t.shape
    ld, step = t.stride()
    if rows <= 1:
        ld = cols
    if (cols > 1 and step != 1) or ld < cols:
        _refuse(t, name, dtypes, index)
    return rows, cols, ld, kind


def _vector(t, name: str, n: int, index: int) -> int:
    """The address of a contiguous binary32 vector of n elements."""
    if not isinstance(t, _Tensor) or not t.is_cuda or t.dtype is not torch.float32:
        raise TypeError(f"{name} must be a float32 tensor on a GPU")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{index}: one call runs on one GPU")
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous vector of {n} elements, not {tuple(t.shape)}")
    return t.data_ptr()


def _run(name: str, index: int, *args) -> None:
    """One entry point of the library on GPU `index`; the stream that is current there comes last."""
    f = getattr(_lib(), name)
    if _current_device() == index:
        rc = f(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = f(*args, _raw_stream(index))
    if rc != PACT_OK:
        raise PactError(rc, name)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(name: str, m: int, n: int, k: int) -> int:
    nbytes = int(getattr(_lib(), name)(m, n, k))
    if nbytes < 0:
        raise PactError(nbytes, name)
    return nbytes


def _scratch(name: str, m: int, n: int, k: int, like: torch.Tensor):
    """(tensor, address, bytes) of scratch for one call: the allocator hands its memory on only to
    later work of the same stream."""
    nbytes = _workspace_bytes(name, m, n, k)
    if nbytes == 0:
        return None, 0, 0
    t = _empty(nbytes, dtype=torch.uint8, device=like.device)
    return t, t.data_ptr(), nbytes


def _by_rows(data: torch.Tensor) -> torch.Tensor:
    """A payload that is not held by rows, in rows of its own."""
    rows, width = data.shape
    if data.dtype is not torch.uint8 or not data.is_cuda or (rows > 1 and data.stride(0) != 1) or data.stride(1) < rows:
        return data.contiguous()
    out = _empty(rows, width, dtype=torch.uint8, device=data.device)
    _run("pact_fp8_transpose", data.get_device(), data.data_ptr(), width, rows, data.stride(1), out.data_ptr(), width)
    return out


class Fp8Matrix:
    """A rows x cols matrix in FP8 with a power-of-two scale for each 128 columns of a row.

    ``data``: uint8 (E4M3 bits), rows x at least cols rounded up to 128, whose columns from
    ``cols`` to that multiple hold zeros; ``scale``: uint8 (biased exponents), rows x at least
    the number of blocks rounded up to four.  Element (i, j) stands for
    ``data[i, j] * 2**(scale[i, j // 128] - 127)``.  ``fp8_quantize`` makes them.  ``data`` whose
    rows are not contiguous (a transposed view, say) is copied into rows that are.
    """

    __slots__ = ("rows", "cols", "_data", "_scale", "_room", "_index", "_bytes")

    def __init__(self, data: torch.Tensor, scale: torch.Tensor, cols: int):
        if isinstance(data, _Tensor) and data.dim() == 2 and data.shape[1] > 1 and data.stride(1) != 1:
            data = _by_rows(data)
        rows, width, ld, _ = _matrix(data, "data", None, _BYTES)
        index = data.get_device()
        scale_rows, scale_width, scale_ld, _ = _matrix(scale, "scale", index, _BYTES)
        cols = int(cols)
        need = (cols + 127) // 128 * 128
        scales = (need // 128 + 3) // 4 * 4
        if cols < 0 or width < need or scale_rows != rows or scale_width < scales:
            raise ValueError(f"data {tuple(data.shape)} and scale {tuple(scale.shape)} do not hold {rows} x {cols} elements")
        self.rows, self.cols, self._data, self._scale, self._room, self._index = rows, cols, data, scale, None, index
        # (one row has no stride of its own, and a matrix without elements none either)
        some = rows > 1 and cols > 0
        self._bytes = _FP8.pack(data.data_ptr(), scale.data_ptr(), rows, cols, ld if some else need,
                                scale_ld if some else scales)

    @staticmethod
    def empty(rows: int, cols: int, device) -> "Fp8Matrix":
        """A matrix of unspecified contents."""
        width = _pad(cols, FP8_BLOCK)
        return Fp8Matrix(torch.empty(rows, width, dtype=torch.uint8, device=device),
                         torch.empty(rows, _pad(width // FP8_BLOCK, 4), dtype=torch.uint8, device=device), cols)

    @staticmethod
    def _sizes(rows: int, cols: int) -> Tuple[int, int, int]:
        """(bytes of a row, scales of a row, where the scales start) in the room of one made by ``_new``."""
        width = (cols + 127) // 128 * 128
        return width, (width // 128 + 3) // 4 * 4, (rows * width + 255) // 256 * 256

    @staticmethod
    def _new(rows: int, cols: int, device, index: int) -> "Fp8Matrix":
        """One of unspecified contents in an allocation of its own; its tensors are made when asked for."""
        m = Fp8Matrix.__new__(Fp8Matrix)
        width, scales, at = Fp8Matrix._sizes(rows, cols)
        room = _empty(at + rows * scales, dtype=torch.uint8, device=device)
        base = room.data_ptr()
        m.rows, m.cols, m._data, m._scale, m._room, m._index = rows, cols, None, None, room, index
        m._bytes = _FP8.pack(base, base + at, rows, cols, width, scales)
        return m

    @property
    def data(self) -> torch.Tensor:
        if self._data is None:
            width, _, _ = self._sizes(self.rows, self.cols)
            self._data = self._room.as_strided((self.rows, width), (width, 1))
        return self._data

    @property
    def scale(self) -> torch.Tensor:
        if self._scale is None:
            _, scales, at = self._sizes(self.rows, self.cols)
            self._scale = self._room.as_strided((self.rows, scales), (scales, 1), at)
        return self._scale

    @property
    def device(self) -> torch.device:
        return (self._data if self._room is None else self._room).device

    @property
    def shape(self) -> Tuple[int, int]:
        return self.rows, self.cols


def _fp8(m, name: str, index=None) -> "Fp8Matrix":
    if not isinstance(m, Fp8Matrix):
        raise TypeError(f"{name} must be an Fp8Matrix")
    if index is not None and m._index != index:
        raise ValueError(f"{name} is on {m.device}, not on cuda:{index}: one call runs on one GPU")
    return m


def fp8_quantize(x: torch.Tensor, along: str = "rows", square: bool = False,
                 out: Union[None, Fp8Matrix, Tuple[Fp8Matrix, Fp8Matrix]] = None):
    """``x`` (rows x cols, float32 or bfloat16) in FP8: ``along`` its "rows" (rows x cols), its
    "columns" (the transposed matrix with its own scales, cols x rows), or "both" in one pass, as
    a pair, each in memory of its own.  ``square``: one scale for each 128 x 128 square (weights).  ``out``: matrices of the
    result's shape to write instead of new ones."""
    rows, cols, ld, kind = _matrix(x, "x")
    if along not in ("rows", "columns", "both"):
        raise ValueError(f"along must be 'rows', 'columns' or 'both', not {along!r}")
    index = x.get_device()
    a = b = None
    if out is None:
        # (each of its own: the columns are kept for the backward pass, and the rows' memory is free before it)
        device = x.device
        if along != "columns":
            a = Fp8Matrix._new(rows, cols, device, index)
        if along != "rows":
            b = Fp8Matrix._new(cols, rows, device, index)
    else:
        a, b = {"rows": (out, None), "columns": (None, out), "both": out}[along]
        for m, want in ((a, (rows, cols)), (b, (cols, rows))):
            if m is not None and _fp8(m, "out", index).shape != want:
                raise ValueError(f"out is {m.shape}, the result is {want}")
    _run("pact_fp8_quantize", index, _MATRIX.pack(x.data_ptr(), rows, cols, ld, kind, 0), None if a is None else a._bytes,
         None if b is None else b._bytes, _FLAG_SQUARE if square else 0)
    if out is not None:
        for m in (a, b):
            if m is not None:
                _changed((m._data, m._scale) if m._room is None else (m._room,))
    return (a, b) if along == "both" else b if a is None else a


def _result(out: Optional[torch.Tensor], rows: int, cols: int, dtype, like, index: int,
            accumulate: bool = False) -> Tuple[torch.Tensor, bytes]:
    """The tensor that a product of rows x cols goes to, and its pact_matrix."""
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs a result to add to")
        if dtype not in _DTYPES:
            raise TypeError(f"the result is float32 or bfloat16, not {dtype}")
        out = _empty(rows, cols, dtype=dtype, device=like.device)
        return out, _MATRIX.pack(out.data_ptr(), rows, cols, cols, _DTYPES[dtype], 0)
    got_rows, got_cols, ld, kind = _matrix(out, "out", index)
    if got_rows != rows or got_cols != cols:
        raise ValueError(f"out is {tuple(out.shape)}, the result is {(rows, cols)}")
    if accumulate and kind != 0:
        raise TypeError("accumulate needs a float32 result")
    return out, _MATRIX.pack(out.data_ptr(), rows, cols, ld, kind, 0)


def fp8_matmul(a: Fp8Matrix, b: Fp8Matrix, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16,
               accumulate: bool = False) -> torch.Tensor:
    """``a @ b.T`` of two FP8 matrices that are quantised along the columns they share: m x n
    elements of ``dtype``, or of ``out``'s; ``accumulate`` adds to ``out`` (float32).  Sums of a
    float32 result are binary32; those of a bfloat16 one are the 8-bit instruction's, a hundredth of
    the result's rounding off."""
    index = _fp8(a, "a")._index
    _fp8(b, "b", index)
    m, n, k = a.rows, b.rows, a.cols
    if k != b.cols:
        raise ValueError(f"a has {k} columns and b {b.cols}")
    given = out is not None
    out, packed = _result(out, m, n, dtype, a, index, accumulate)
    _keep, at, nbytes = _scratch("pact_fp8_matmul_workspace_bytes", m, n, k, a)
    _run("pact_fp8_matmul", index, a._bytes, b._bytes, packed, _FLAG_ACCUMULATE if accumulate else 0, at, nbytes)
    if given:
        _changed((out,))
    return out


def fp8_linear(x: torch.Tensor, w: Fp8Matrix, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16) -> torch.Tensor:
    """``x @ W.T``: ``x`` (float32 or bfloat16) quantised along its rows and multiplied by ``w``."""
    rows, cols, ld, kind = _matrix(x, "x")
    index = x.get_device()
    n = _fp8(w, "w", index).rows
    if cols != w.cols:
        raise ValueError(f"x has {cols} columns and w {w.cols}")
    given = out is not None
    out, packed = _result(out, rows, n, dtype, x, index)
    _keep, at, nbytes = _scratch("pact_fp8_linear_workspace_bytes", rows, n, cols, x)
    _run("pact_fp8_linear", index, _MATRIX.pack(x.data_ptr(), rows, cols, ld, kind, 0), w._bytes, packed, at, nbytes)
    if given:
        _changed((out,))
    return out


def fp8_linear_backward(dy: torch.Tensor, w_columns: Fp8Matrix, x_columns: Fp8Matrix,
                        grad_weight: Optional[torch.Tensor] = None, accumulate: bool = False,
                        need_dx: bool = True) -> Tuple[Optional[torch.Tensor], torch.Tensor]:
    """The gradients of ``y = x W^T`` from ``dy`` (rows x n): ``(dx, dw)`` with ``dx = dy W`` in dy's
    type and ``dw = dy^T x`` in float32, written or (``accumulate``) added to ``grad_weight``.
    (Where dx's sums cancel below 2^-6 of their terms, hand dy over in float32: binary32 sums for both.)

    ``w_columns`` and ``x_columns``: W (n x k) and x (rows x k) quantised along their columns, so
    k x n and k x rows.  ``need_dx=False`` leaves dx out (None)."""
    m, n, ld, kind = _matrix(dy, "dy")
    index = dy.get_device()
    k = _fp8(x_columns, "x_columns", index).rows
    _fp8(w_columns, "w_columns", index)
    if x_columns.cols != m:
        raise ValueError(f"dy has {m} rows and x {x_columns.cols}")
    if w_columns.cols != n or w_columns.rows != k:
        raise ValueError(f"w_columns is {w_columns.shape}, not {(k, n)}")
    if grad_weight is not None and (not isinstance(grad_weight, _Tensor) or grad_weight.dtype is not torch.float32):
        raise TypeError("grad_weight must be a float32 tensor")
    dw, dw_packed = _result(grad_weight, n, k, torch.float32, dy, index, accumulate)
    dx, dx_packed = _result(None, m, k, dy.dtype, dy, index) if need_dx else (None, None)
    _keep, at, nbytes = _scratch("pact_fp8_linear_backward_workspace_bytes", m, n, k, dy)
    _run("pact_fp8_linear_backward", index, _MATRIX.pack(dy.data_ptr(), m, n, ld, kind, 0), w_columns._bytes,
         x_columns._bytes, dx_packed, dw_packed, _FLAG_ACCUMULATE if accumulate else 0, at, nbytes)
    if grad_weight is not None:
        _changed((dw,))
    return dx, dw


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

def _distill(name: str, logits, top_logits, top_index, temperature, row_weight, grad, lse, keep_lse: bool):
    """One call of the loss, the gradient (from ``lse``) or both: (loss, lse, grad) as far as it makes them.
    ``grad``: False for none, None for a new one."""
    rows, vocab, ld, kind = _matrix(logits, "logits")
    index = logits.get_device()
    t_rows, top, t_ld, t_kind = _matrix(top_logits, "top_logits", index)
    i_rows, i_top, i_ld, i_bytes = _matrix(top_index, "top_index", index, _INDEX)
    if t_rows != rows or i_rows != rows or i_top != top:
        raise ValueError(f"logits {tuple(logits.shape)}, top_logits {tuple(top_logits.shape)} and top_index "
                         f"{tuple(top_index.shape)} do not go together")
    if top > DISTILL_MAX_TOP:
        raise ValueError(f"at most {DISTILL_MAX_TOP} of the teacher's logits a row, not {top}")
    weight_at = 0 if row_weight is None else _vector(row_weight, "row_weight", rows, index)
    loss = None
    lse_at = loss_at = grad_at = grad_ld = 0
    if lse is not None:
        lse_at = _vector(lse, "lse", rows, index)
    else:
        loss = _empty(rows, dtype=torch.float32, device=logits.device)
        loss_at = loss.data_ptr()
        if keep_lse:  # (of its own: parting one allocation costs more than a second)
            lse = _empty(rows, dtype=torch.float32, device=logits.device)
            lse_at = lse.data_ptr()
    given = None
    if grad is None:
        grad = _empty(rows, vocab, dtype=logits.dtype, device=logits.device)
        grad_at, grad_ld = grad.data_ptr(), vocab
    elif grad is not False:
        g_rows, g_cols, grad_ld, g_kind = _matrix(grad, "grad", index)
        if g_rows != rows or g_cols != vocab or g_kind != kind:
            raise ValueError(f"grad must be {logits.dtype} of {tuple(logits.shape)}")
        grad_at, given = grad.data_ptr(), grad
    try:
        packed = _DISTILL.pack(logits.data_ptr(), grad_at, top_logits.data_ptr(), top_index.data_ptr(), weight_at, loss_at,
                               lse_at, rows, vocab, top, ld, grad_ld, t_ld, i_ld, temperature, kind, t_kind, i_bytes, 0,
                               _raw_stream(index))
    except struct.error:
        raise TypeError(f"temperature must be a number, not {temperature!r}") from None
    except OverflowError:  # (beyond binary32, as infinity is)
        raise PactError(PACT_EINVAL, name) from None
    f = getattr(_lib(), name)
    if _current_device() == index:
        rc = f(packed)
    else:
        with torch.cuda.device(index):
            rc = f(packed)
    if rc != PACT_OK:
        raise PactError(rc, name)
    if given is not None:
        _changed((given,))
    return loss, lse, grad


def distill_loss(logits: torch.Tensor, top_logits: torch.Tensor, top_index: torch.Tensor, temperature: float = 1.0,
                 row_weight: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``(loss, lse)``, float32 vectors: each row's weighted Kullback-Leibler divergence of the student
    (``logits``, rows x vocab) from the teacher's softmax over its listed logits (``top_logits`` and
    their ``top_index``, rows x top; a negative index is an empty slot), and the log-sum-exp of
    ``logits / temperature`` that ``distill_grad`` takes."""
    loss, lse, _ = _distill("pact_distill_loss", logits, top_logits, top_index, temperature, row_weight, False, None, True)
    return loss, lse


def distill_grad(logits: torch.Tensor, top_logits: torch.Tensor, top_index: torch.Tensor, lse: torch.Tensor,
                 temperature: float = 1.0, row_weight: Optional[torch.Tensor] = None,
                 grad: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``distill_loss`` for the logits, in their type.  ``row_weight``: the loss's, times
    the upstream gradient of each row's loss.  ``grad``: where to write it; may be ``logits``."""
    if lse is None:
        raise TypeError("lse must be the second result of distill_loss")
    return _distill("pact_distill_grad", logits, top_logits, top_index, temperature, row_weight, grad, lse, False)[2]


def distill_step(logits: torch.Tensor, top_logits: torch.Tensor, top_index: torch.Tensor, temperature: float = 1.0,
                 row_weight: Optional[torch.Tensor] = None,
                 grad: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``(loss, grad)`` of one training step, the logits read once where a row fits a workgroup's registers
    (up to 32768 entries of bfloat16, 65536 of float32) and twice, mostly from the caches, where it is longer.
    ``grad`` may be ``logits``: the gradient then takes their place."""
    loss, _, grad = _distill("pact_distill_step", logits, top_logits, top_index, temperature, row_weight, grad, None, False)
    return loss, grad
