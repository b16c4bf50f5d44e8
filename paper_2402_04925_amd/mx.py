"""Microscaled (MX) operands: 4-bit floating-point weights and 8- or 4-bit
activations with one power-of-two scale per 32 elements (include/tpdq.h).

As in the rest of the binding, every function only marshals torch tensors into the
C ABI. A result that the caller gives no buffer for, and a workspace, come from
torch's allocator within the call, on the device's current stream.
"""
from __future__ import annotations

import ctypes
import dataclasses
from typing import Optional

from . import _abi
from . import Workspace, _dtype_code, _stream_handle, _torch
from ._abi import MX_FP4, MX_FP8, MX_ROWS, MX_TILED

_BLOCK, _STEP, _CHUNK, _TILE = 32, 128, 512, 32


def _up(a: int, b: int) -> int:
    return -(-a // b)


def _on(device):
    """Makes the tensors' device current for the launch where it is not."""
    torch = _torch()
    if device.index is None or device.index == torch.cuda.current_device():
        return None
    return torch.cuda.device(device)


def _run(device, f, *args):
    guard = _on(device)
    if guard is None:
        _abi.check(f(*args, _stream_handle(device)))
    else:
        with guard:
            _abi.check(f(*args, _stream_handle(device)))


def _gpu(t, name):
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a GPU, got {t.device}")


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, X on {device}")


def _rows16(name, t, shape=None, dtype=None):
    """A 16-bit matrix with unit column stride (of this shape and type)."""
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


@dataclasses.dataclass
class MxTensor:
    """An R x K tensor of MX numbers in device memory (or a shard of one as views).

    MX_ROWS: codes [R][>= padded K], float8_e4m3fn (fp8) or uint8 with two codes
    to a byte (fp4); scale_bytes uint8 [R][>= padded blocks]. MX_TILED (weights):
    codes uint8 [ceil(R/32)][...], scale_bytes uint8 [ceil(R/32)][...], the order that
    mx_gemm reads (see include/tpdq.h). Rows are padded to whole steps (codes, 128
    elements) and chunks (scales, 512 elements), with zeros."""
    codes: object
    scale_bytes: object
    R: int
    K: int
    fmt: int
    layout: int = MX_ROWS

    @classmethod
    def empty(cls, R: int, K: int, fmt: int, device, layout: int = MX_ROWS) -> "MxTensor":
        """Storage for mx_quantize, rmsnorm or mx_pack to write."""
        torch = _torch()
        if fmt not in (MX_FP4, MX_FP8):
            raise ValueError(f"unknown format {fmt}")
        steps, chunks = _up(K, _STEP), _up(K, _CHUNK)
        if layout == MX_TILED:
            rows, c, s = _up(R, _TILE), steps * 2048, chunks * 512
        else:
            rows, c, s = R, steps * (64 if fmt == MX_FP4 else 128), chunks * 16
        t = torch.float8_e4m3fn if fmt == MX_FP8 else torch.uint8
        return cls(torch.empty((rows, c), dtype=t, device=device),
                   torch.empty((rows, s), dtype=torch.uint8, device=device), R, K, fmt, layout)

    @classmethod
    def from_tensors(cls, codes, scales, K: int, fmt: int) -> "MxTensor":
        """An MX_ROWS tensor from dense codes ([R][ceil(K/32) * 32] fp8, half as
        many bytes for fp4) and scales ([R][ceil(K/32)], uint8 or float8_e8m0fnu),
        copied into padded rows. Codes at and past K count as zeros."""
        torch = _torch()
        blocks, R = _up(K, _BLOCK), codes.shape[0]
        per = 16 if fmt == MX_FP4 else 32
        if K < 1 or K % 8 or tuple(codes.shape) != (R, blocks * per) or tuple(scales.shape) != (R, blocks):
            raise ValueError(f"K={K} (a multiple of 8) takes codes [R][{blocks * per}] and scales [R][{blocks}], got "
                             f"{list(codes.shape)} and {list(scales.shape)}")
        q = cls.empty(R, K, fmt, codes.device)
        c = q.codes.view(torch.uint8)
        used = K // 2 if fmt == MX_FP4 else K
        c[:, :used] = codes.view(torch.uint8)[:, :used]
        c[:, used:] = 0
        q.scale_bytes[:, :blocks] = scales.view(torch.uint8)
        q.scale_bytes[:, blocks:] = 0
        return q

    @property
    def device(self):
        return self.codes.device

    @property
    def scales(self):
        """MX_ROWS: the scales' values, float8_e8m0fnu [R][ceil(K/32)]."""
        torch = _torch()
        if self.layout != MX_ROWS:
            raise ValueError("a tiled tensor has no scales by rows")
        return self.scale_bytes[:, :_up(self.K, _BLOCK)].view(torch.float8_e8m0fnu)

    def c_struct(self) -> _abi.Mx:
        torch = _torch()
        c, s = self.codes, self.scale_bytes
        if (c.dim() != 2 or s.dim() != 2 or c.stride(1) != 1 or s.stride(1) != 1 or c.device != s.device
                or c.dtype is not (torch.float8_e4m3fn if self.fmt == MX_FP8 else torch.uint8)
                or s.dtype is not torch.uint8 or c.shape[0] != s.shape[0]
                or c.shape[0] != (self.R if self.layout == MX_ROWS else _up(self.R, _TILE))):
            raise ValueError("codes and scale_bytes must be 2-D with unit column stride, on one device, a row for each "
                             "row (tiled: each 32), of float8_e4m3fn (fp8) or uint8 (fp4) and of uint8")
        _gpu(c, "an MX tensor")
        # rows further apart than their number of rows asks for: one row has any stride
        ld_c = c.stride(0) if c.shape[0] > 1 else c.shape[1]
        ld_s = s.stride(0) if s.shape[0] > 1 else s.shape[1]
        return _abi.Mx(c.data_ptr(), ld_c, s.data_ptr(), ld_s, self.R, self.K, self.fmt, self.layout)

    def column_shard(self, rank: int, tp: int) -> "MxTensor":
        """Column-parallel share of a weight (views): outputs [rank*R/tp, ...)."""
        n = self.R // tp
        r0 = rank * n
        if self.layout == MX_TILED:
            if n % _TILE and tp > 1:
                raise ValueError("a tiled column shard must start and end on 32-row tiles")
            a, b = r0 // _TILE, _up(r0 + n, _TILE)
        else:
            a, b = r0, r0 + n
        return MxTensor(self.codes[a:b], self.scale_bytes[a:b], n, self.K, self.fmt, self.layout)

    def row_shard(self, rank: int, tp: int) -> "MxTensor":
        """Row-parallel share of a weight (views): inputs [rank*K/tp, ...)."""
        k = self.K // tp
        if k % _CHUNK and tp > 1:
            raise ValueError("a row shard must start and end on multiples of 512 inputs")
        if tp == 1:
            return self
        steps, chunks = k // _STEP, k // _CHUNK
        per_c, per_s = (2048, 512) if self.layout == MX_TILED else (64 if self.fmt == MX_FP4 else 128, 16)
        return MxTensor(self.codes[:, rank * steps * per_c:(rank + 1) * steps * per_c],
                        self.scale_bytes[:, rank * chunks * per_s:(rank + 1) * chunks * per_s],
                        self.R, k, self.fmt, self.layout)


def mx_quantize(X, fmt: int, out: Optional[MxTensor] = None) -> MxTensor:
    """X [R][K] (fp16 or bf16, K a multiple of 8) in MX numbers of format fmt."""
    _rows16("X", X)
    _gpu(X, "X")
    if out is None:
        out = MxTensor.empty(X.shape[0], X.shape[1], fmt, X.device)
    elif (out.R, out.K, out.fmt, out.layout) != (X.shape[0], X.shape[1], fmt, MX_ROWS):
        raise ValueError("out must have X's shape, the format asked for and the MX_ROWS layout")
    _same_device(X.device, out=out)
    cq = out.c_struct()
    _run(X.device, _abi.lib().tpdq_mx_quantize, X.data_ptr(), X.stride(0), _dtype_code(X.dtype), ctypes.byref(cq))
    return out


def mx_dequantize(q: MxTensor, dtype, out=None):
    """The values of an MX_ROWS tensor, rounded once to fp16 or bf16."""
    torch = _torch()
    if out is None:
        out = torch.empty((q.R, q.K), dtype=dtype, device=q.device)
    _rows16("out", out, (q.R, q.K), dtype)
    _same_device(q.device, out=out)
    cq = q.c_struct()
    _run(q.device, _abi.lib().tpdq_mx_dequantize, ctypes.byref(cq), _dtype_code(dtype), out.data_ptr(), out.stride(0))
    return out


def mx_pack(q: MxTensor) -> MxTensor:
    """An fp4 weight [N][K] in the order that the products read (offline)."""
    out = MxTensor.empty(q.R, q.K, q.fmt, q.device, MX_TILED)
    a, b = q.c_struct(), out.c_struct()
    _run(q.device, _abi.lib().tpdq_mx_pack, ctypes.byref(a), ctypes.byref(b))
    return out


def rmsnorm(X, weight, eps: float, residual=None, fmt: Optional[int] = None, residual_out=None, out=None):
    """h = X + residual (rounded to X's type; X itself without one), y = h /
    sqrt(mean(h^2) + eps) * weight. Returns (y, h): y in X's type, or with fmt
    as an MxTensor; h in residual_out (which may be residual itself) or new."""
    torch = _torch()
    _rows16("X", X)
    _gpu(X, "X")
    M, K = X.shape
    dev = X.device
    if weight.dim() != 1 or weight.shape[0] != K or not weight.is_contiguous():
        raise ValueError(f"weight must be a contiguous [{K}]")
    if weight.dtype != X.dtype:
        raise TypeError(f"weight is {weight.dtype}, X is {X.dtype}: one element type per call")
    h, ldr, ldh = X, 0, 0
    if residual is not None:
        _rows16("residual", residual, (M, K), X.dtype)
        h = torch.empty((M, K), dtype=X.dtype, device=dev) if residual_out is None else residual_out
        _rows16("residual_out", h, (M, K), X.dtype)
        ldr, ldh = residual.stride(0), h.stride(0)
    elif residual_out is not None:
        raise ValueError("residual_out needs a residual")
    y = cq = None
    if fmt is None:
        y = torch.empty((M, K), dtype=X.dtype, device=dev) if out is None else out
        _rows16("out", y, (M, K), X.dtype)
    else:
        out = MxTensor.empty(M, K, fmt, dev) if out is None else out
        if not isinstance(out, MxTensor) or (out.R, out.K, out.fmt, out.layout) != (M, K, fmt, MX_ROWS):
            raise ValueError("out must be an MxTensor of X's shape, the format asked for and the MX_ROWS layout")
        cq = out.c_struct()
    _same_device(dev, weight=weight, residual=residual, residual_out=h, out=out if y is None else y)
    _run(dev, _abi.lib().tpdq_rmsnorm, X.data_ptr(), X.stride(0), None if residual is None else residual.data_ptr(), ldr,
         weight.data_ptr(), eps, M, K, _dtype_code(X.dtype), None if residual is None else h.data_ptr(), ldh,
         None if y is None else y.data_ptr(), 0 if y is None else y.stride(0), None if cq is None else ctypes.byref(cq))
    return (out if y is None else y), h


def _scratch(workspace: Optional[Workspace], nbytes: int, device):
    """The caller's workspace, or one of the call's own: calls that are captured
    in two graphs, or run on two streams, share none."""
    torch = _torch()
    if workspace is not None:
        return workspace.get(nbytes)
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def mx_gemm(X: MxTensor, w: MxTensor, dtype, out=None, workspace: Optional[Workspace] = None):
    """Y = X W^T: X [M][K] fp8 or fp4, w [N][K] fp4 from mx_pack, fp32 accumulation,
    Y [M][N] rounded once to dtype."""
    torch = _torch()
    dev = X.device
    _same_device(dev, w=w, out=out)
    if out is None:
        out = torch.empty((X.R, w.R), dtype=dtype, device=dev)
    _rows16("out", out, (X.R, w.R), dtype)
    cx, cw = X.c_struct(), w.c_struct()
    lib = _abi.lib()
    nbytes = lib.tpdq_mx_workspace_bytes(_abi.OP_MX_GEMM, X.R, ctypes.byref(cw), None)
    buf = _scratch(workspace, nbytes, dev)
    _run(dev, lib.tpdq_mx_gemm, ctypes.byref(cx), ctypes.byref(cw), _dtype_code(dtype), out.data_ptr(), out.stride(0),
         None if buf is None else buf.data_ptr(), 0 if buf is None else buf.numel())
    return out


def mx_mlp_shard(X: MxTensor, w_up: MxTensor, w_down: MxTensor, dtype, w_gate: Optional[MxTensor] = None, out=None,
                 workspace: Optional[Workspace] = None):
    """One rank's MLP share up to the AllReduce: Y1 = X W_up^T, or silu(X W_gate^T)
    * (X W_up^T) with w_gate, quantized in X's format; returns Y2_partial = Y1
    W_down^T. w_up and w_gate are column shards, w_down a row shard."""
    torch = _torch()
    dev = X.device
    _same_device(dev, w_up=w_up, w_down=w_down, w_gate=w_gate, out=out)
    if out is None:
        out = torch.empty((X.R, w_down.R), dtype=dtype, device=dev)
    _rows16("out", out, (X.R, w_down.R), dtype)
    if X.R > 1 and out.stride(0) != w_down.R:
        raise ValueError("out must be dense")
    cx, cu, cd = X.c_struct(), w_up.c_struct(), w_down.c_struct()
    cg = None if w_gate is None else w_gate.c_struct()
    lib = _abi.lib()
    nbytes = lib.tpdq_mx_workspace_bytes(_abi.OP_MX_MLP, X.R, ctypes.byref(cu), ctypes.byref(cd))
    buf = _scratch(workspace, nbytes, dev)
    _run(dev, lib.tpdq_mx_mlp_shard, ctypes.byref(cx), None if cg is None else ctypes.byref(cg), ctypes.byref(cu),
         ctypes.byref(cd), _dtype_code(dtype), out.data_ptr(), None if buf is None else buf.data_ptr(),
         0 if buf is None else buf.numel())
    return out
