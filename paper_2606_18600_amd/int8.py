"""Products in 8-bit integers over torch tensors (``stage_quant_*`` of the ABI).

``quantize`` turns the rows of a matrix into 8-bit integers with a scale each:
activations before a product, or weights once, when they are loaded
(``pack_weight`` takes weights that are in 8 bits already). ``product`` multiplies
two of them, ``linear`` quantises activations and multiplies in one call::

    w = int8.quantize(weight)            # [n, k] bf16 or fp32, once
    y = int8.linear(x, w)                # [..., k] -> [..., n]

A quantised weight [vocab, hidden] also serves as the LM head's
(``harness.DeviceStage.lm_head``). Everything runs on torch's current stream of
the tensors' device; outputs and scratch come from torch's allocator, so calls
may be captured into a graph.
"""

from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import stage as S

DTYPES = {torch.float32: S.STAGE_F32, torch.bfloat16: S.STAGE_BF16}


def invalid(msg: str) -> S.StageError:
    return S.StageError(S.STAGE_ERR_INVALID_ARG, msg)


def unsupported(msg: str) -> S.StageError:
    return S.StageError(S.STAGE_ERR_UNSUPPORTED, msg)


def on_gpu(*tensors: Optional[torch.Tensor]) -> torch.device:
    """The GPU that all the tensors (None aside) are on."""
    device = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise invalid(f"a tensor is on {t.device}, not on a GPU")
        if device is None:
            device = t.device
        elif t.device != device:
            raise invalid(f"tensors on {device} and {t.device}")
    return device


class at_device:
    """Makes ``device`` current, where it is not, for the calls of a block and
    gives torch's current stream on it."""

    __slots__ = ("device", "guard")

    def __init__(self, device: torch.device):
        self.device, self.guard = device, None

    def __enter__(self) -> int:
        if torch.cuda.current_device() != self.device.index:
            self.guard = torch.cuda.device(self.device)
            self.guard.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *exc) -> None:
        if self.guard is not None:
            self.guard.__exit__(*exc)


def rows_of(x: torch.Tensor, what: str) -> torch.Tensor:
    """x as [rows, k] with adjacent values in a row."""
    if x.dim() == 0:
        raise invalid(f"{what} has no dimension")
    if x.dim() != 2:
        x = x.reshape(-1, x.shape[-1])
    if x.shape[1] > 1 and x.stride(1) != 1:
        x = x.contiguous()
    elif x.shape[0] > 1 and x.stride(0) < x.shape[1]:
        x = x.contiguous()  # rows that overlap (an expanded tensor)
    return x


def row_stride(x: torch.Tensor) -> int:
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


@dataclass(frozen=True)
class Matrix:
    """A quantised [rows, k] matrix: opaque device memory of its values and
    scales."""

    data: torch.Tensor
    rows: int
    k: int

    @property
    def shape(self):
        return (self.rows, self.k)


def _empty(rows: int, k: int, device) -> torch.Tensor:
    n = S.stage_quant_bytes(rows, k)
    if n == 0 and rows > 0:
        raise S.StageError(S.STAGE_ERR_UNSUPPORTED, S.stage_last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)


def quantize(x: torch.Tensor) -> Matrix:
    """The rows [..., k] of x (fp32 or bf16) in 8 bits, each by its largest
    magnitude."""
    dt = DTYPES.get(x.dtype)
    if dt is None:
        raise unsupported(f"quantize: {x.dtype}")
    device = on_gpu(x)
    x = rows_of(x, "x")
    m, k = x.shape
    with at_device(device) as stream:
        data = _empty(m, k, device)
        S.stage_quant_rows(dt, x.data_ptr(), row_stride(x), m, k, data.data_ptr(), stream)
    return Matrix(data, m, k)


def pack_weight(values: torch.Tensor, scales: torch.Tensor) -> Matrix:
    """Weights that are in 8 bits already: values [n, k] int8, scales [n] fp32."""
    if values.dim() != 2 or values.dtype != torch.int8:
        raise invalid("pack_weight: values must be int8 [n, k]")
    if scales.dtype != torch.float32 or scales.shape != values.shape[:1]:
        raise invalid("pack_weight: scales must be float32 [n]")
    device = on_gpu(values, scales)
    values, scales = rows_of(values, "values"), scales.contiguous()
    n, k = values.shape
    with at_device(device) as stream:
        data = _empty(n, k, device)
        S.stage_quant_pack(values.data_ptr(), row_stride(values), scales.data_ptr(), n, k,
                           data.data_ptr(), stream)
    return Matrix(data, n, k)


def product(a: Matrix, b: Matrix, dtype: torch.dtype = torch.bfloat16,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T [a.rows, b.rows] in ``dtype``, or into ``out`` (any row stride)."""
    if a.k != b.k:
        raise invalid(f"product of {a.shape} and {b.shape}")
    device = on_gpu(a.data, b.data, out)
    if out is not None:
        dtype = out.dtype
        if out.shape != (a.rows, b.rows) or (out.numel() and b.rows > 1 and out.stride(1) != 1) or \
                (a.rows > 1 and out.stride(0) < b.rows):
            raise invalid(f"product: out {tuple(out.shape)} with strides {out.stride()}")
    dt = DTYPES.get(dtype)
    if dt is None:
        raise unsupported(f"product: {dtype}")
    with at_device(device) as stream:
        if out is None:
            out = torch.empty((a.rows, b.rows), dtype=dtype, device=device)
        size = S.stage_quant_product_bytes(a.rows, b.rows, a.k)
        ws = torch.empty(size, dtype=torch.uint8, device=device) if size else None
        S.stage_quant_product(a.data.data_ptr(), a.rows, b.data.data_ptr(), b.rows, a.k, dt,
                              out.data_ptr(), row_stride(out),
                              None if ws is None else ws.data_ptr(), size, stream)
    return out


def linear(x: torch.Tensor, w: Matrix, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """x [..., k] (fp32 or bf16) times w [n, k] transposed: [..., n] in ``dtype``
    (x's own unless given)."""
    if x.dim() == 0 or x.shape[-1] != w.k:
        raise invalid(f"linear: {tuple(x.shape)} times {w.shape}")
    on_gpu(x, w.data)
    y = product(quantize(x), w, x.dtype if dtype is None else dtype)
    return y if x.dim() == 2 else y.view(*x.shape[:-1], w.rows)
