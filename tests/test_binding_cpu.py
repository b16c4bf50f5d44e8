"""What the binding refuses on the host, before the library is called (no GPU)."""
import gc
import types
import weakref

import pytest
import torch

import paper_2402_04925_amd as tpdq
from paper_2402_04925_amd import mx

GPU = torch.device("cuda", 0)  # named, not used


# ---- workspaces ----------------------------------------------------------

TAKERS = [lambda ws: tpdq._workspace(GPU, 100, ws), lambda ws: mx._scratch(ws, 100, GPU)]


@pytest.mark.parametrize("take", TAKERS)
def test_workspace_of_another_device_is_refused(take):
    """Kernels write the workspace: host memory, or another GPU's, must not reach them."""
    with pytest.raises(ValueError, match="workspace"):
        take(tpdq.Workspace("cpu"))
    used = tpdq.Workspace()
    used.get(10)  # on torch's default device, here the CPU
    with pytest.raises(ValueError, match="workspace"):
        take(used)


@pytest.mark.parametrize("take", TAKERS)
def test_workspace_without_a_device_takes_the_call_s(take, monkeypatch):
    made, host = [], torch.zeros(1 << 20, dtype=torch.uint8)

    def empty(*size, dtype, device):
        made.append(device)
        return host

    monkeypatch.setattr(torch, "empty", empty)
    ws = tpdq.Workspace()
    with pytest.raises(ValueError, match="workspace"):  # the stand-in's memory is no GPU's
        take(ws)
    assert made == [GPU] and ws.device == GPU


# ---- MxTensor.from_tensors -----------------------------------------------

U8, E8M0 = torch.uint8, torch.float8_e8m0fnu
CODES = {tpdq.MX_FP8: ([torch.float8_e4m3fn, U8], 64), tpdq.MX_FP4: ([U8, torch.float4_e2m1fn_x2], 32)}


def ones(dtype, *shape):
    """Bytes 1 of a one-byte type, ones of any other."""
    if dtype.itemsize == 1:
        return torch.ones(*shape, dtype=U8).view(dtype)
    return torch.ones(*shape, dtype=dtype)


@pytest.mark.parametrize("fmt", [tpdq.MX_FP4, tpdq.MX_FP8])
def test_from_tensors_takes_the_format_s_types(fmt):
    types, n = CODES[fmt]
    for t in types:
        for s in (U8, E8M0):
            q = tpdq.MxTensor.from_tensors(ones(t, 2, n), ones(s, 2, 2), 64, fmt)
            assert (q.codes.view(U8)[:, :n] == 1).all() and (q.scales.view(U8) == 1).all()


@pytest.mark.parametrize("fmt", [tpdq.MX_FP4, tpdq.MX_FP8])
def test_from_tensors_refuses_other_types(fmt):
    """Their bytes are no codes of the format: a float's, an int32's, another fp8's."""
    types, n = CODES[fmt]
    others = [torch.float8_e4m3fnuz, torch.float8_e5m2, torch.int8, torch.bool, torch.float16, torch.int32, torch.float32,
              torch.int64] + ([torch.float8_e4m3fn] if fmt == tpdq.MX_FP4 else [torch.float4_e2m1fn_x2])
    for t in others:
        with pytest.raises(TypeError):
            tpdq.MxTensor.from_tensors(ones(t, 2, n), ones(U8, 2, 2), 64, fmt)
    for t in (torch.int8, torch.bool, torch.float8_e4m3fn, torch.float16, torch.float32, torch.int32):
        with pytest.raises(TypeError):
            tpdq.MxTensor.from_tensors(ones(types[0], 2, n), ones(t, 2, 2), 64, fmt)


def test_from_tensors_refuses_two_devices():
    with pytest.raises(ValueError, match="device|on "):
        tpdq.MxTensor.from_tensors(ones(U8, 2, 64), torch.empty(2, 2, dtype=U8, device="meta"), 64, tpdq.MX_FP8)


# ---- counts past the C ABI's 32 bits -------------------------------------

MANY = (1 << 32) + 8  # 8 in its low 32 bits


def meta(*shape, dtype=torch.float16):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("layout", [tpdq.MX_ROWS, tpdq.MX_TILED])
@pytest.mark.parametrize("R,K", [(MANY, 8), (8, MANY), (1 << 31, 8), (8, 1 << 31)])
def test_mx_sizes_past_32_bits_are_refused(R, K, layout):
    with pytest.raises(ValueError, match="2\\^31"):
        tpdq.MxTensor.empty(R, K, tpdq.MX_FP4, "meta", layout)
    rows = R if layout == tpdq.MX_ROWS else -(-R // 32)
    per_c, per_s = tpdq.MxTensor._widths(tpdq.MX_FP4, layout)
    with pytest.raises(ValueError, match="2\\^31"):
        tpdq.MxTensor(meta(rows, -(-K // 128) * per_c, dtype=U8), meta(rows, -(-K // 512) * per_s, dtype=E8M0), R, K,
                      tpdq.MX_FP4, layout)


def test_largest_mx_size_is_kept():
    q = tpdq.MxTensor.empty((1 << 31) - 1, 8, tpdq.MX_FP4, "meta")
    assert (q._c.R, q._c.K) == ((1 << 31) - 1, 8)


@pytest.mark.parametrize("shape", [(MANY, 8), (8, MANY)])
def test_16_bit_rows_past_32_bits_are_refused(shape):
    x = meta(*shape)
    with pytest.raises(ValueError, match="2\\^31"):
        tpdq.rmsnorm(x, meta(shape[1]), 1e-5)
    with pytest.raises(ValueError, match="2\\^31"):
        tpdq.mx_quantize(x, tpdq.MX_FP8)


def test_w4a16_counts_past_32_bits_are_refused():
    x = types.SimpleNamespace(device=GPU, shape=(MANY, 8), dtype=torch.float16)
    with pytest.raises(ValueError, match="2\\^31"):
        tpdq._check_args(GPU, torch.float16, X=x)
    for K, N in ((MANY, 8), (8, MANY)):
        w = tpdq.QuantWeight.from_tensors(meta(K // 8, N, dtype=torch.int32), meta(1, N), meta(1, N // 8, dtype=torch.int32),
                                          None, K, 1)
        with pytest.raises(ValueError, match="2\\^31"):
            w.c_struct()
    w = tpdq.QuantWeight.from_tensors(meta(1, 8, dtype=torch.int32), meta(1, 8), meta(1, 1, dtype=torch.int32), None, 8, 1)
    with pytest.raises(ValueError, match="2\\^31"):
        tpdq.workspace_bytes(tpdq.OP_GEMM, MANY, w)


def test_outgrown_buffers_are_kept():
    """A captured graph still writes the buffer that its calls were given."""
    ws = tpdq.Workspace("cpu")
    first = weakref.ref(ws.get(100))
    assert ws.get(8 << 20).numel() >= 8 << 20 and ws.get(100) is ws.buf
    gc.collect()
    assert first() is not None
    # and they stay few: each is at least twice the one before
    ws, seen = tpdq.Workspace("cpu"), set()
    for n in range(1 << 20, 16 << 20, 1 << 16):
        b = ws.get(n)
        seen.add((b.data_ptr(), b.numel()))
    assert len(seen) <= 5 and sum(n for _, n in seen) < 2 * b.numel()
