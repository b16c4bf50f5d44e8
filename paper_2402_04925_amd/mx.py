"""Microscaled (MX) operands: 4-bit floating-point weights and 8- or 4-bit
activations with one power-of-two scale per 32 elements (include/tpdq.h).

As in the rest of the binding, every function only marshals torch tensors into the
C ABI. A result that the caller gives no buffer for, and a workspace, come from
torch's allocator within the call, on the device's current stream.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

from . import _abi
from . import Workspace, _dtype_code, _stream_handle, _torch, _workspace
from ._abi import MX_FP4, MX_FP8, MX_ROWS, MX_TILED

_BLOCK, _STEP, _CHUNK, _TILE = 32, 128, 512, 32


def _up(a: int, b: int) -> int:
    return -(-a // b)


def _run(device, f, *args):
    """f(*args, stream) with the tensors' device current (a launch needs that)."""
    cuda = _torch().cuda
    if device.index is None or device.index == cuda.current_device():
        st = f(*args, _stream_handle(device))
    else:
        with cuda.device(device):
            st = f(*args, _stream_handle(device))
    if st:
        _abi.check(st)


def _device_of(name, t):
    dev = t.device
    if dev.type != "cuda":
        raise ValueError(f"{name} must be on a GPU, got {dev}")
    return dev


def _same_device(device, name, t):
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, X on {device}")


def _ld(t):
    """Leading dimension of a matrix; one row has whatever stride, and is its length apart."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _rows16(name, t, M=None, K=None, dtype=None):
    """A 16-bit matrix with unit column stride (M x K, of dtype)."""
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    if M is None and (t.shape[0] > _abi.COUNT_MAX or t.shape[1] > _abi.COUNT_MAX):
        _abi.check_counts(rows=t.shape[0], columns=t.shape[1])
    if M is not None and (t.shape[0] != M or t.shape[1] != K):
        raise ValueError(f"{name} must be [{M}][{K}], got {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


class MxTensor:
    """An R x K tensor of MX numbers in device memory (or a shard of one as views).
    Its fields are not assigned anew: the C struct that calls pass is made once.

    MX_ROWS: codes [R][>= padded K], float8_e4m3fn (fp8) or uint8 with two codes
    to a byte (fp4); padded_scales float8_e8m0fnu [R][>= padded blocks]. MX_TILED
    (weights): codes uint8 [ceil(R/32)][...], padded_scales [ceil(R/32)][...], the order
    that mx_gemm reads (see include/tpdq.h). Rows are padded to whole steps (codes,
    128 elements) and chunks (scales, 512 elements), with zero bytes."""

    __slots__ = ("_codes", "_scales", "_R", "_K", "_fmt", "_layout", "_device", "_c", "_ref")

    def __init__(self, codes, padded_scales, R: int, K: int, fmt: int, layout: int = MX_ROWS):
        torch = _torch()
        _abi.check_counts(R=R, K=K)
        c, s = codes, padded_scales
        rows = R if layout == MX_ROWS else _up(R, _TILE)
        dev = c.device
        if (c.dim() != 2 or s.dim() != 2 or c.stride(1) != 1 or s.stride(1) != 1 or s.device != dev
                or c.dtype is not (torch.float8_e4m3fn if fmt == MX_FP8 else torch.uint8)
                or s.dtype is not torch.float8_e8m0fnu or c.shape[0] != rows or s.shape[0] != rows):
            raise ValueError("codes (float8_e4m3fn for fp8, uint8 for fp4) and padded_scales (float8_e8m0fnu) must be 2-D "
                             "with unit column stride, on one device, a row for each row (tiled: each 32)")
        # the C ABI sees the leading dimensions alone: columns cut short may end past the storage
        per_c, per_s = self._widths(fmt, layout)
        if c.shape[1] < _up(K, _STEP) * per_c or s.shape[1] < _up(K, _CHUNK) * per_s:
            raise ValueError(f"rows of {c.shape[1]} bytes of codes and {s.shape[1]} scales are shorter than K={K} padded to "
                             f"whole steps and chunks")
        self._set(c, s, R, K, fmt, layout, dev, _ld(c), _ld(s))

    @staticmethod
    def _widths(fmt, layout):
        """Bytes of a row (of a tile): of codes per step, of scales per chunk."""
        if fmt not in (MX_FP4, MX_FP8):
            raise ValueError(f"unknown format {fmt}")
        return (2048, 512) if layout == MX_TILED else (64 if fmt == MX_FP4 else 128, 16)

    def _set(self, c, s, R, K, fmt, layout, dev, ld_c, ld_s):
        self._codes, self._scales, self._R, self._K, self._fmt, self._layout, self._device = c, s, R, K, fmt, layout, dev
        self._c = _abi.Mx(c.data_ptr(), ld_c, s.data_ptr(), ld_s, R, K, fmt, layout)
        self._ref = ctypes.byref(self._c)

    codes = property(lambda self: self._codes)
    padded_scales = property(lambda self: self._scales)
    R = property(lambda self: self._R)
    K = property(lambda self: self._K)
    fmt = property(lambda self: self._fmt)
    layout = property(lambda self: self._layout)
    device = property(lambda self: self._device)

    @classmethod
    def empty(cls, R: int, K: int, fmt: int, device, layout: int = MX_ROWS) -> "MxTensor":
        """Storage for mx_quantize, rmsnorm or mx_pack to write. (Sizes go to torch apart: as
        a tuple an allocation takes 1.6 us, so 1.3.)"""
        torch = _torch()
        if R > _abi.COUNT_MAX or K > _abi.COUNT_MAX:
            _abi.check_counts(R=R, K=K)
        per_c, per_s = cls._widths(fmt, layout)
        c, s = -(-K // _STEP) * per_c, -(-K // _CHUNK) * per_s
        t = torch.float8_e4m3fn if fmt == MX_FP8 else torch.uint8
        rows = -(-R // _TILE) if layout == MX_TILED else R
        q = cls.__new__(cls)
        codes = torch.empty(rows, c, dtype=t, device=device)
        q._set(codes, torch.empty(rows, s, dtype=torch.float8_e8m0fnu, device=device), R, K, fmt, layout, codes.device,
               c, s)
        return q

    @classmethod
    def from_tensors(cls, codes, scales, K: int, fmt: int) -> "MxTensor":
        """An MX_ROWS tensor from dense codes ([R][ceil(K/32) * 32] fp8, float8_e4m3fn
        or its bytes as uint8; half as many bytes for fp4, uint8 or float4_e2m1fn_x2)
        and scales ([R][ceil(K/32)], uint8 or float8_e8m0fnu), copied into padded rows.
        Codes at and past K count as zeros."""
        torch = _torch()
        own = {MX_FP8: torch.float8_e4m3fn, MX_FP4: getattr(torch, "float4_e2m1fn_x2", torch.uint8)}
        if fmt not in own:
            raise ValueError(f"unknown format {fmt}")
        if codes.dtype not in (torch.uint8, own[fmt]) or scales.dtype not in (torch.uint8, torch.float8_e8m0fnu):
            raise TypeError(f"codes must be uint8 or {own[fmt]} and scales uint8 or float8_e8m0fnu, got {codes.dtype} and "
                            f"{scales.dtype}")
        if scales.device != codes.device:
            raise ValueError(f"scales are on {scales.device}, codes on {codes.device}")
        blocks, R = _up(K, _BLOCK), codes.shape[0]
        per = 16 if fmt == MX_FP4 else 32
        if K < 1 or K % 8 or tuple(codes.shape) != (R, blocks * per) or tuple(scales.shape) != (R, blocks):
            raise ValueError(f"K={K} (a multiple of 8) takes codes [R][{blocks * per}] and scales [R][{blocks}], got "
                             f"{list(codes.shape)} and {list(scales.shape)}")
        q = cls.empty(R, K, fmt, codes.device)
        c, s = q.codes.view(torch.uint8), q.padded_scales.view(torch.uint8)
        used = K // 2 if fmt == MX_FP4 else K
        c[:, :used] = codes.view(torch.uint8)[:, :used]
        c[:, used:] = 0
        s[:, :blocks] = scales.view(torch.uint8)
        s[:, blocks:] = 0
        return q

    @property
    def scales(self):
        """MX_ROWS: the scales' values, float8_e8m0fnu [R][ceil(K/32)]."""
        if self._layout != MX_ROWS:
            raise ValueError("a tiled tensor has no scales by rows")
        n = -(-self._K // _BLOCK)
        return self._scales if self._scales.shape[1] == n else self._scales[:, :n]

    def column_shard(self, rank: int, tp: int) -> "MxTensor":
        """Column-parallel share of a weight (views): outputs [rank*R/tp, ...)."""
        n = self._R // tp
        if n * tp != self._R or not 0 <= rank < tp:
            raise ValueError(f"rank {rank} of {tp} has no equal share of {self._R} outputs")
        r0 = rank * n
        if self._layout == MX_TILED:
            if n % _TILE and tp > 1:
                raise ValueError("a tiled column shard must start and end on 32-row tiles")
            a, b = r0 // _TILE, _up(r0 + n, _TILE)
        else:
            a, b = r0, r0 + n
        return MxTensor(self._codes[a:b], self._scales[a:b], n, self._K, self._fmt, self._layout)

    def row_shard(self, rank: int, tp: int) -> "MxTensor":
        """Row-parallel share of a weight (views): inputs [rank*K/tp, ...)."""
        k = self._K // tp
        if k * tp != self._K or not 0 <= rank < tp:
            raise ValueError(f"rank {rank} of {tp} has no equal share of {self._K} inputs")
        if k % _CHUNK and tp > 1:
            raise ValueError("a row shard must start and end on multiples of 512 inputs")
        if tp == 1:
            return self
        steps, chunks = k // _STEP, k // _CHUNK
        per_c, per_s = self._widths(self._fmt, self._layout)
        return MxTensor(self._codes[:, rank * steps * per_c:(rank + 1) * steps * per_c],
                        self._scales[:, rank * chunks * per_s:(rank + 1) * chunks * per_s],
                        self._R, k, self._fmt, self._layout)


def _mx_arg(name, q, device=None):
    if not isinstance(q, MxTensor):
        raise TypeError(f"{name} must be an MxTensor, got {type(q).__name__}")
    if q._device.type != "cuda":
        raise ValueError(f"{name} must be on a GPU, got {q._device}")
    if device is not None and q._device != device:
        raise ValueError(f"{name} is on {q._device}, X on {device}")
    return q._ref


def _mx_out(out, M, K, fmt, device):
    if out is None:
        return MxTensor.empty(M, K, fmt, device)
    _mx_arg("out", out, device)
    if (out._R, out._K, out._fmt, out._layout) != (M, K, fmt, MX_ROWS):
        raise ValueError("out must be an MxTensor of X's shape, the format asked for and the MX_ROWS layout")
    return out


def mx_quantize(X, fmt: int, out: Optional[MxTensor] = None) -> MxTensor:
    """X [R][K] (fp16 or bf16, K a multiple of 8) in MX numbers of format fmt."""
    _rows16("X", X)
    dev = _device_of("X", X)
    out = _mx_out(out, X.shape[0], X.shape[1], fmt, dev)
    _run(dev, _abi.lib().tpdq_mx_quantize, X.data_ptr(), _ld(X), _dtype_code(X.dtype), out._ref)
    return out


def mx_dequantize(q: MxTensor, dtype, out=None):
    """The values of an MX_ROWS tensor, rounded once to fp16 or bf16."""
    ref = _mx_arg("q", q)
    dev = q._device
    code = _dtype_code(dtype)
    if out is None:
        out = _torch().empty(q._R, q._K, dtype=dtype, device=dev)
    else:
        _rows16("out", out, q._R, q._K, dtype)
        _same_device(dev, "out", out)
    _run(dev, _abi.lib().tpdq_mx_dequantize, ref, code, out.data_ptr(), _ld(out))
    return out


def mx_pack(q: MxTensor) -> MxTensor:
    """An fp4 weight [N][K] in the order that the products read (offline)."""
    ref = _mx_arg("q", q)
    out = MxTensor.empty(q._R, q._K, q._fmt, q._device, MX_TILED)
    _run(q._device, _abi.lib().tpdq_mx_pack, ref, out._ref)
    return out


def rmsnorm(X, weight, eps: float, residual=None, fmt: Optional[int] = None, residual_out=None, out=None):
    """h = X + residual (rounded to X's type; X itself without one), y = h /
    sqrt(mean(h^2) + eps) * weight. Returns (y, h): y in X's type, or with fmt
    as an MxTensor; h in residual_out or new. residual_out and out may each be X or
    residual itself; memory shared otherwise is refused."""
    torch = _torch()
    _rows16("X", X)
    dev, dt = _device_of("X", X), X.dtype
    M, K = X.shape
    code = _dtype_code(dt)
    if weight.dim() != 1 or weight.shape[0] != K or not weight.is_contiguous():
        raise ValueError(f"weight must be a contiguous [{K}]")
    if weight.dtype != dt:
        raise TypeError(f"weight is {weight.dtype}, X is {dt}: one element type per call")
    _same_device(dev, "weight", weight)
    h, res, ldr, hp, ldh = X, None, 0, None, 0
    if residual is not None:
        _rows16("residual", residual, M, K, dt)
        _same_device(dev, "residual", residual)
        if residual_out is None:
            h = torch.empty(M, K, dtype=dt, device=dev)
        else:
            h = residual_out
            _rows16("residual_out", h, M, K, dt)
            _same_device(dev, "residual_out", h)
        res, ldr, hp, ldh = residual.data_ptr(), _ld(residual), h.data_ptr(), _ld(h)
    elif residual_out is not None:
        raise ValueError("residual_out needs a residual")
    if fmt is None:
        if out is None:
            out = torch.empty(M, K, dtype=dt, device=dev)
        else:
            _rows16("out", out, M, K, dt)
            _same_device(dev, "out", out)
        y, ldy, ref = out.data_ptr(), _ld(out), None
    else:
        out = _mx_out(out, M, K, fmt, dev)
        y, ldy, ref = None, 0, out._ref
    _run(dev, _abi.lib().tpdq_rmsnorm, X.data_ptr(), _ld(X), res, ldr, weight.data_ptr(), eps, M, K, code, hp, ldh,
         y, ldy, ref)
    return out, h


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(op: int, M: int, R: int, K: int, R2: int) -> int:
    """tpdq_mx_workspace_bytes: of the sizes alone."""
    a = _abi.Mx(None, 0, None, 0, R, K, MX_FP4, MX_TILED)
    b = _abi.Mx(None, 0, None, 0, R2, R, MX_FP4, MX_TILED)
    return _abi.lib().tpdq_mx_workspace_bytes(op, M, ctypes.byref(a), ctypes.byref(b) if R2 else None)


def _scratch(workspace: Optional[Workspace], nbytes: int, device):
    """(address, bytes) and the tensor that holds it: the caller's workspace, or one
    of the call's own, so that calls captured in two graphs, or running on two
    streams, share none."""
    if not nbytes:
        return None, 0, None
    if workspace is None:
        buf = _torch().empty(nbytes, dtype=_torch().uint8, device=device)
    else:
        buf = _workspace(device, nbytes, workspace)
    return buf.data_ptr(), buf.numel(), buf


def _out16(out, M, N, dtype, device):
    if out is None:
        return _torch().empty(M, N, dtype=dtype, device=device)
    _rows16("out", out, M, N, dtype)
    _same_device(device, "out", out)
    return out


def mx_gemm(X: MxTensor, w: MxTensor, dtype, out=None, workspace: Optional[Workspace] = None):
    """Y = X W^T: X [M][K] fp8 or fp4, w [N][K] fp4 from mx_pack, Y [M][N] rounded once to
    dtype. fp32 accumulation; of each 8 consecutive products with an fp8 X, what lies 13
    bits below the largest is dropped (about 1e-4 of a typical output)."""
    cx = _mx_arg("X", X)
    dev = X._device
    cw = _mx_arg("w", w, dev)
    code = _dtype_code(dtype)
    out = _out16(out, X._R, w._R, dtype, dev)
    ws, nbytes, _buf = _scratch(workspace, _workspace_bytes(_abi.OP_MX_GEMM, X._R, w._R, w._K, 0), dev)
    _run(dev, _abi.lib().tpdq_mx_gemm, cx, cw, code, out.data_ptr(), _ld(out), ws, nbytes)
    return out


def mx_mlp_shard(X: MxTensor, w_up: MxTensor, w_down: MxTensor, dtype, w_gate: Optional[MxTensor] = None, out=None,
                 workspace: Optional[Workspace] = None):
    """One rank's MLP share up to the AllReduce: Y1 = X W_up^T, or silu(X W_gate^T)
    * (X W_up^T) with w_gate, quantized in X's format; returns Y2_partial = Y1
    W_down^T. w_up and w_gate are column shards, w_down a row shard. Sums as in
    mx_gemm; what an fp8 X loses there can change codes of Y1 (see include/tpdq.h)."""
    cx = _mx_arg("X", X)
    dev = X._device
    cu, cd = _mx_arg("w_up", w_up, dev), _mx_arg("w_down", w_down, dev)
    cg = None if w_gate is None else _mx_arg("w_gate", w_gate, dev)
    code = _dtype_code(dtype)
    if w_down._K != w_up._R:
        raise ValueError(f"w_down takes {w_down._K} inputs, w_up has {w_up._R} outputs")
    out = _out16(out, X._R, w_down._R, dtype, dev)
    if X._R > 1 and out.stride(0) != w_down._R:
        raise ValueError("out must be dense")
    ws, nbytes, _buf = _scratch(workspace, _workspace_bytes(_abi.OP_MX_MLP, X._R, w_up._R, w_up._K, w_down._R), dev)
    _run(dev, _abi.lib().tpdq_mx_mlp_shard, cx, cg, cu, cd, code, out.data_ptr(), ws, nbytes)
    return out
