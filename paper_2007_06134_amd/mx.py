"""Microscaled messages on torch tensors: the ``adpsgd_mx_*`` calls of ``include/adpsgd.h``.

What a worker sends at a synchronization is its difference from the model that
all workers share, in 4 (E2M1) or 8 bits (E4M3) an element, blocks of 32
elements sharing a power of two.  Every function runs on the current stream of
its tensors' device, waits for nothing and can be captured into a graph;
outputs and workspaces that the caller does not pass come from torch's
allocator.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from ._native import MX_E2M1, MX_E4M3, _check, adpsgd_mx_rows, lib

BLOCK = 32                            # elements that share a scale
_ROW_BYTES = {MX_E2M1: 16, MX_E4M3: 32}   # of codes, a block


class MxRows:
    """K rows of P elements: codes [K, >= ceil(P / 32) * 16 (E2M1) or * 32 (E4M3)] and scales
    [K, >= ceil(P / 32)], uint8, rows at strides that are multiples of 16 bytes."""

    __slots__ = ("codes", "scales", "P", "format", "K", "_c")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, P: int, format: int = MX_E2M1):
        if format not in _ROW_BYTES:
            raise ValueError("format must be MX_E2M1 or MX_E4M3")
        if P < 0:
            raise ValueError("P must be >= 0")
        n = -(-P // BLOCK)
        for t, need, name in ((codes, n * _ROW_BYTES[format], "codes"), (scales, n, "scales")):
            if t.dtype != torch.uint8 or t.dim() != 2 or t.device.type != "cuda":
                raise ValueError(f"{name} must be a uint8 matrix on a GPU")
            if t.shape[1] < need or (t.shape[1] > 1 and t.stride(1) != 1):
                raise ValueError(f"{name} must have rows of at least {need} contiguous bytes")
        if codes.shape[0] != scales.shape[0] or codes.device != scales.device:
            raise ValueError("codes and scales must have one row a worker on one device")
        self.codes, self.scales, self.P, self.format, self.K = codes, scales, P, format, codes.shape[0]
        self._c = adpsgd_mx_rows(codes.data_ptr(), scales.data_ptr(), _row_stride(codes, 16), _row_stride(scales, 16),
                                 P, self.K, format)

    @classmethod
    def empty(cls, K: int, P: int, format: int = MX_E2M1, device="cuda") -> "MxRows":
        """Rows to be written, at adpsgd_mx_code_stride and adpsgd_mx_scale_stride."""
        if format not in _ROW_BYTES:
            raise ValueError("format must be MX_E2M1 or MX_E4M3")
        if K < 1 or P < 0:
            raise ValueError("K must be >= 1 and P >= 0")
        opt = dict(dtype=torch.uint8, device=device)
        return cls(torch.empty((K, lib.adpsgd_mx_code_stride(format, P)), **opt),
                   torch.empty((K, lib.adpsgd_mx_scale_stride(P)), **opt), P, format)

    @property
    def device(self) -> torch.device:
        return self.codes.device


def _row_stride(t: torch.Tensor, unit: int) -> int:
    """Distance of rows; of a single row or empty ones, whose stride means nothing, their length in whole units."""
    return t.stride(0) if t.shape[0] > 1 and t.shape[1] > 0 else -(-t.shape[1] // unit) * unit


def _matrix(t: torch.Tensor, K: int, P: int, device, name: str) -> int:
    """Row stride of a float32 [K, P] tensor."""
    if t.dtype != torch.float32 or t.shape != (K, P) or t.device != device:
        raise ValueError(f"{name} must be float32 [{K}, {P}] on {device}")
    if P > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if K > 1 and t.stride(0) < P:
        raise ValueError(f"{name} must have rows that do not overlap")
    return t.stride(0) if K > 1 else P


def _vector(t: Optional[torch.Tensor], P: int, device, name: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (P,) or t.device != device or (P > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be contiguous float32 [{P}] on {device}")
    return t.data_ptr()


def _offsets(t: torch.Tensor, device) -> int:
    if t.dtype != torch.int64 or t.dim() != 1 or t.shape[0] < 2 or t.device != device or t.stride(0) != 1:
        raise ValueError(f"offsets must be contiguous int64 [T + 1] on {device}")
    return t.shape[0] - 1


class _On:
    """The device of a call made current, and its current stream."""

    __slots__ = ("guard",)

    def __init__(self, device):
        self.guard = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def mx_quantize(x: torch.Tensor, base: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, *,
                format: Optional[int] = None, residual_out: Optional[torch.Tensor] = None,
                out: Optional[MxRows] = None) -> MxRows:
    """The messages of the K workers whose parameters are x [K, P]: (x - base) + residual in `format`.

    base [P] and residual [K, P] count as zero where they are None.  What the message leaves out is
    written to residual_out, by default to residual itself, and not kept where both are None.
    out: rows to write (their format is the one used)."""
    if x.dim() != 2 or x.device.type != "cuda":
        raise ValueError("x must be a float32 matrix on a GPU")
    K, P = x.shape
    device = x.device
    x_ld = _matrix(x, K, P, device, "x")
    base_ptr = _vector(base, P, device, "base")
    if residual_out is None:
        residual_out = residual
    r_in = r_out = None
    r_ld = 0
    if residual_out is not None:
        r_ld, r_out = _matrix(residual_out, K, P, device, "residual_out"), residual_out.data_ptr()
    if residual is not None:
        if _matrix(residual, K, P, device, "residual") != r_ld:
            raise ValueError("residual and residual_out must have the same row stride")
        r_in = residual.data_ptr()
    if out is None:
        out = MxRows.empty(K, P, MX_E2M1 if format is None else format, device)
    elif out.K != K or out.P != P or out.device != device or (format is not None and format != out.format):
        raise ValueError(f"out must be rows of the format for [{K}, {P}] on {device}")
    with _On(device) as stream:
        _check(lib.adpsgd_mx_quantize(C.byref(out._c), x.data_ptr(), x_ld, base_ptr, r_in, r_out, r_ld, stream))
    return out


def mx_dequantize(rows: MxRows, base: Optional[torch.Tensor] = None, *,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """What the rows say: base + their values, float32 [K, P]."""
    device = rows.device
    base_ptr = _vector(base, rows.P, device, "base")
    if out is None:
        out = torch.empty((rows.K, rows.P), dtype=torch.float32, device=device)
    ld = _matrix(out, rows.K, rows.P, device, "out")
    with _On(device) as stream:
        _check(lib.adpsgd_mx_dequantize(C.byref(rows._c), base_ptr, out.data_ptr(), ld, stream))
    return out


def mx_average(rows: MxRows, offsets: torch.Tensor, base: Optional[torch.Tensor] = None, *,
               x: Optional[torch.Tensor] = None,
               base_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The synchronization: (base + the rows' mean, float32 [P]; every tensor's variance, float64 [T]).

    offsets: int64 [T + 1] on the device, the tensors' boundaries as for ``Adpsgd`` (0 first, P last;
    the values are not checked).  The new model is also written to every row of x [K, P] where that is
    given, and to base_out (which may be base; a new tensor by default)."""
    device = rows.device
    T = _offsets(offsets, device)
    base_ptr = _vector(base, rows.P, device, "base")
    x_ptr, x_ld = None, 0
    if x is not None:
        x_ld, x_ptr = _matrix(x, rows.K, rows.P, device, "x"), x.data_ptr()
    if base_out is None:
        base_out = torch.empty((rows.P,), dtype=torch.float32, device=device)
    out_ptr = _vector(base_out, rows.P, device, "base_out")
    var = torch.empty((T,), dtype=torch.float64, device=device)
    need = lib.adpsgd_mx_average_workspace(rows.K, rows.P, T)
    work = torch.empty((need,), dtype=torch.uint8, device=device)
    with _On(device) as stream:
        _check(lib.adpsgd_mx_average(C.byref(rows._c), T, offsets.data_ptr(), base_ptr, out_ptr, x_ptr, x_ld,
                                     var.data_ptr(), work.data_ptr(), need, stream))
    return base_out, var


def mx_product(a: MxRows, offsets: torch.Tensor, b: Optional[MxRows] = None) -> torch.Tensor:
    """Inner products of the rows of a with those of b (of a, where b is None) for every tensor:
    float32 [T, K, K].  K is at most 256; a and b have the same format, K and P."""
    device = a.device
    T = _offsets(offsets, device)
    if b is not None and b.device != device:
        raise ValueError("a and b must be on one device")
    out = torch.empty((T, a.K, a.K), dtype=torch.float32, device=device)
    need = lib.adpsgd_mx_product_workspace(a.K, a.P, T)
    work = torch.empty((need,), dtype=torch.uint8, device=device)
    with _On(device) as stream:
        _check(lib.adpsgd_mx_product(C.byref(a._c), None if b is None else C.byref(b._c), T, offsets.data_ptr(),
                                     out.data_ptr(), work.data_ptr(), need, stream))
    return out
