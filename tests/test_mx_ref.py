"""The MX reference (tests/mx_ref.py) against brute force, and the C ABI's refusals
of malformed MX calls (no call here reaches a kernel launch)."""
import ctypes
import os

import numpy as np
import pytest

from paper_2402_04925_amd import _abi
from tests import mx_ref as ref

needs_no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake device pointers only where no GPU exists")


@pytest.mark.parametrize("fmt", [ref.FP4, ref.FP8])
def test_nearest_is_the_closest_value_ties_to_even(fmt):
    t = ref.table(fmt)
    assert t[-1] == (6 if fmt == ref.FP4 else 448) and (np.diff(t) > 0).all()
    mids = (t[1:] + t[:-1]) / 2
    a = np.concatenate([t, mids, np.nextafter(mids, 0), np.nextafter(mids, 1e9), [t[-1] * 1.3],
                        np.random.default_rng(1).uniform(0, t[-1], 2000)])
    for x, c in zip(a, ref.nearest(a, fmt)):
        d = np.abs(t - x)
        best = np.flatnonzero(d == d.min())
        assert c in best and (len(best) == 1 or c % 2 == 0), (x, c)


def test_fp8_table_is_torch_float8():
    import torch
    b = torch.arange(256, dtype=torch.uint8)
    want = b.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.elements(b.numpy(), ref.FP8), want)


@pytest.mark.parametrize("fmt", [ref.FP4, ref.FP8])
def test_quantize_by_hand(fmt):
    top = 2 if fmt == ref.FP4 else 8
    x = np.zeros((1, 72))
    x[0, :32] = 2.0 ** 10            # scale 2^(10 - top), code of 2^top
    x[0, 33] = -3 * 2.0 ** -127      # scale at its smallest
    x[0, 64] = np.inf
    c, s = ref.quantize(x, fmt)
    assert s.tolist() == [[127 + 10 - top, max(0, -126 - top + 127), 255]]
    assert (ref.elements(c[0, :32], fmt) == 2.0 ** top).all() and c[0, 64] == 0
    assert ref.values(c, s, fmt)[0, 33] == (-3 * 2.0 ** -127 if fmt == ref.FP8 else -3 * 2.0 ** -127)
    assert np.isnan(ref.values(c, s, fmt)[0, 64:]).all()


def test_tiled_places_every_code_once():
    N, K = 40, 136
    codes = np.random.default_rng(2).integers(1, 16, (N, K)).astype(np.uint8)
    c, s = ref.tiled(codes, np.full((N, 5), 9, np.uint8))
    nib = np.stack([c & 15, c >> 4], -1).reshape(-1)
    assert (np.bincount(nib, minlength=16)[1:] == np.bincount(codes.reshape(-1), minlength=16)[1:]).all()
    assert (s == 9).sum() == N * 5 and (s != 0).sum() == N * 5


def test_the_gpu_tests_reach_every_kernel(lib):
    """The products that tests/test_gpu_mx.py runs, by the kernel that is planned for
    them: every tile shape in 16 bits, quantized and gated, and splits of K."""
    from tests import test_gpu_mx as t
    plan = getattr(lib, "_ZN4tpdq7plan_mxEiiiibb")  # MxPlan plan_mx(M, N, K, fmt, gated, quant)
    plan.restype, plan.argtypes = ctypes.c_int64, [ctypes.c_int] * 4 + [ctypes.c_bool] * 2
    rows, half, t128x512, t64x512, t64x256, t128x256, t64x128, t64x64 = range(8)
    for fmt in (ref.FP4, ref.FP8):
        seen = {}
        for gated, quant in ((False, False), (False, True), (True, True)):
            for M, N, K in t.TILES + ([] if quant else t.SHAPES + t.LARGE):
                p = plan(M, N, K, fmt, gated, quant)
                seen.setdefault((gated, quant), set()).add((p & 0xFFFFFFFF, (p >> 32) > 1))
        tiles = {t128x512, t64x512, t64x256, t128x256, t64x128, t64x64}
        assert {k for k, _ in seen[False, False]} == tiles | {rows, half}
        assert {k for k, _ in seen[False, True]} == tiles | {rows}
        assert {k for k, _ in seen[True, True]} == tiles - {t64x64} | {rows}
        assert all(any(split for _, split in kinds) for kinds in seen.values())
        assert {(t64x128, False), (t64x128, True)} <= seen[True, True]  # two groups of waves


# ---- refusals ------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_abi.LIB_PATH):
        from paper_2402_04925_amd import build
        build.build()
    return _abi.lib()


def rows(R=4, K=256, fmt=_abi.MX_FP8, base=1 << 24, **kw):
    d = dict(codes=base, ld_c=-(-K // 128) * (64 if fmt == _abi.MX_FP4 else 128), scales=base + (1 << 22),
             ld_s=-(-K // 512) * 16, R=R, K=K, format=fmt, layout=_abi.MX_ROWS)
    return _abi.Mx(**{**d, **kw})


def tiled(N=64, K=256, base=1 << 26, **kw):
    d = dict(codes=base, ld_c=-(-K // 128) * 2048, scales=base + (1 << 22), ld_s=-(-K // 512) * 512, R=N, K=K,
             format=_abi.MX_FP4, layout=_abi.MX_TILED)
    return _abi.Mx(**{**d, **kw})


def ref_of(q):
    return None if q is None else ctypes.byref(q)


BAD_ROWS = [
    (dict(codes=None), _abi.ERR_NULL), (dict(scales=None), _abi.ERR_NULL), (dict(format=2), _abi.ERR_SHAPE),
    (dict(layout=_abi.MX_TILED), _abi.ERR_SHAPE), (dict(layout=5), _abi.ERR_SHAPE), (dict(R=0), _abi.ERR_SHAPE),
    (dict(R=-1), _abi.ERR_SHAPE), (dict(K=0), _abi.ERR_SHAPE), (dict(K=252), _abi.ERR_SHAPE),
    (dict(ld_c=128), _abi.ERR_SHAPE), (dict(ld_s=0), _abi.ERR_SHAPE), (dict(ld_c=264), _abi.ERR_ALIGN),
    (dict(ld_s=24), _abi.ERR_ALIGN), (dict(codes=(1 << 24) + 8), _abi.ERR_ALIGN),
    (dict(scales=(1 << 25) + 4), _abi.ERR_ALIGN),
]


@needs_no_gpu
@pytest.mark.parametrize("change,want", BAD_ROWS)
def test_bad_rows_tensor_is_refused(lib, change, want):
    q = rows(**change)
    assert lib.tpdq_mx_quantize(1 << 30, 256, 0, ref_of(q), None) == want
    assert lib.tpdq_mx_dequantize(ref_of(q), 0, 1 << 30, 256, None) == want
    assert lib.tpdq_rmsnorm(1 << 30, 256, None, 0, 1 << 31, 1e-5, 4, 256, 0, None, 0, None, 0, ref_of(q), None) == want
    w = tiled()
    assert lib.tpdq_mx_gemm(ref_of(q), ref_of(w), 0, 1 << 30, 64, 1 << 28, 1 << 30, None) == want
    d = tiled(N=96, K=64, base=1 << 27)
    assert lib.tpdq_mx_mlp_shard(ref_of(q), None, ref_of(w), ref_of(d), 0, 1 << 30, 1 << 28, 1 << 30, None) == want


@needs_no_gpu
def test_quantize_refusals(lib):
    q = rows()
    f = lambda X=1 << 30, ldx=256, dt=0, t=q: lib.tpdq_mx_quantize(X, ldx, dt, ref_of(t), None)
    assert f(X=None) == _abi.ERR_NULL and f(t=None) == _abi.ERR_NULL
    assert f(ldx=248) == _abi.ERR_SHAPE and f(dt=2) == _abi.ERR_SHAPE
    assert f(X=(1 << 30) + 8) == _abi.ERR_ALIGN and f(ldx=260) == _abi.ERR_ALIGN
    assert f(t=rows(R=1 << 30, K=8192)) == _abi.ERR_SHAPE  # ldx < K
    assert f(t=rows(R=1 << 30, K=8192), ldx=8192) == _abi.ERR_UNSUPPORTED
    # five chunks of a row are two workgroups of three waves: 2^32 threads from 2^28 / 6 rows on
    assert f(t=rows(R=(1 << 28) // 5 - 1, K=2056), ldx=2056) == _abi.ERR_UNSUPPORTED
    assert f(t=rows(R=(1 << 28) - 1, K=8), ldx=8) == _abi.ERR_UNSUPPORTED
    g = lambda X=1 << 30, ldx=256, dt=0: lib.tpdq_mx_dequantize(ref_of(q), dt, X, ldx, None)
    assert g(X=None) == _abi.ERR_NULL and g(ldx=128) == _abi.ERR_SHAPE and g(dt=-1) == _abi.ERR_SHAPE
    assert g(X=(1 << 30) + 2) == _abi.ERR_ALIGN


@needs_no_gpu
def test_pack_refusals(lib):
    src, dst = rows(R=64, fmt=_abi.MX_FP4), tiled()
    f = lambda a=src, b=dst: lib.tpdq_mx_pack(ref_of(a), ref_of(b), None)
    assert f(a=None) == _abi.ERR_NULL and f(b=None) == _abi.ERR_NULL
    assert f(a=rows(R=64)) == _abi.ERR_UNSUPPORTED                      # fp8 weights
    assert f(b=tiled(format=_abi.MX_FP8)) == _abi.ERR_UNSUPPORTED
    assert f(b=tiled(N=96)) == _abi.ERR_SHAPE and f(b=tiled(K=384)) == _abi.ERR_SHAPE
    assert f(b=tiled(ld_c=2048)) == _abi.ERR_SHAPE and f(b=tiled(ld_s=256)) == _abi.ERR_SHAPE
    assert f(b=tiled(ld_s=520)) == _abi.ERR_ALIGN
    assert f(a=dst, b=dst) == _abi.ERR_SHAPE
    huge = 1 << 28
    assert f(a=rows(R=huge, fmt=_abi.MX_FP4), b=tiled(N=huge)) == _abi.ERR_UNSUPPORTED


@needs_no_gpu
def test_rmsnorm_refusals(lib):
    def f(X=1 << 30, ldx=256, res=None, ldr=256, w=1 << 31, eps=1e-5, M=4, K=256, dt=0, h=None, ldh=256, Y=1 << 32,
          ldy=256, q=None):
        return lib.tpdq_rmsnorm(X, ldx, res, ldr, w, eps, M, K, dt, h, ldh, Y, ldy, ref_of(q), None)
    assert f(X=None) == _abi.ERR_NULL and f(w=None) == _abi.ERR_NULL
    assert f(res=1 << 33) == _abi.ERR_NULL and f(h=1 << 33) == _abi.ERR_NULL     # both or none
    assert f(Y=None) == _abi.ERR_NULL and f(q=rows()) == _abi.ERR_NULL           # one output
    assert f(M=0) == _abi.ERR_SHAPE and f(K=0) == _abi.ERR_SHAPE and f(K=252) == _abi.ERR_SHAPE
    assert f(dt=3) == _abi.ERR_SHAPE and f(eps=-1.0) == _abi.ERR_SHAPE and f(eps=float("nan")) == _abi.ERR_SHAPE
    assert f(K=65544, ldx=65544, ldy=65544) == _abi.ERR_UNSUPPORTED
    assert f(ldx=128) == _abi.ERR_SHAPE and f(ldy=128) == _abi.ERR_SHAPE
    assert f(ldx=260) == _abi.ERR_ALIGN and f(w=(1 << 31) + 8) == _abi.ERR_ALIGN and f(Y=(1 << 32) + 8) == _abi.ERR_ALIGN
    r = dict(res=1 << 33, h=1 << 34)
    assert f(**r, ldr=128) == _abi.ERR_SHAPE and f(**r, ldh=128) == _abi.ERR_SHAPE and f(**r, ldr=260) == _abi.ERR_ALIGN
    assert f(**{**r, "h": 1 << 32}) == _abi.ERR_SHAPE                             # Y and residual_out are one
    big = dict(M=1 << 22, K=8192, ldx=8192, ldy=8192)
    assert f(**big) == _abi.ERR_UNSUPPORTED                                       # 2^32 threads
    assert f(Y=None, q=rows(R=5)) == _abi.ERR_SHAPE and f(Y=None, q=rows(K=384)) == _abi.ERR_SHAPE


@needs_no_gpu
def test_product_refusals(lib):
    def f(x=rows(), w=tiled(), dt=0, Y=1 << 30, ldy=64):
        return lib.tpdq_mx_gemm(ref_of(x), ref_of(w), dt, Y, ldy, 1 << 28, 1 << 30, None)
    assert f(x=None) == _abi.ERR_NULL and f(w=None) == _abi.ERR_NULL and f(Y=None) == _abi.ERR_NULL
    assert f(dt=2) == _abi.ERR_SHAPE and f(ldy=56) == _abi.ERR_SHAPE
    assert f(w=tiled(N=60)) == _abi.ERR_SHAPE and f(w=tiled(K=384)) == _abi.ERR_SHAPE
    assert f(w=rows(R=64, fmt=_abi.MX_FP4)) == _abi.ERR_SHAPE                    # not packed
    assert f(Y=(1 << 30) + 8) == _abi.ERR_ALIGN and f(ldy=68) == _abi.ERR_ALIGN
    assert f(x=rows(R=1 << 23)) == _abi.ERR_UNSUPPORTED                          # 2 GiB of codes
    assert f(x=rows(ld_c=1 << 31, R=1)) == _abi.ERR_UNSUPPORTED
    big = (1 << 30) + 8
    assert f(x=rows(R=1, K=big), w=tiled(K=big)) == _abi.ERR_UNSUPPORTED         # longer rows than any call takes
    assert f(w=tiled(ld_c=1 << 30)) == _abi.ERR_UNSUPPORTED


@needs_no_gpu
def test_mlp_refusals(lib):
    up, down = tiled(N=96), tiled(N=64, K=96, base=1 << 27)
    need = lib.tpdq_mx_workspace_bytes(_abi.OP_MX_MLP, 4, ref_of(up), ref_of(down))
    assert need > 0

    def f(x=rows(), g=None, u=up, d=down, dt=0, Y=1 << 30, ws=1 << 28, nb=need):
        return lib.tpdq_mx_mlp_shard(ref_of(x), ref_of(g), ref_of(u), ref_of(d), dt, Y, ws, nb, None)
    assert f(u=None) == _abi.ERR_NULL and f(d=None) == _abi.ERR_NULL and f(Y=None) == _abi.ERR_NULL
    assert f(d=tiled(N=64, K=104)) == _abi.ERR_SHAPE                             # K2 != N1
    assert f(g=tiled(N=64)) == _abi.ERR_SHAPE and f(g=tiled(N=96, ld_c=8192)) == _abi.ERR_SHAPE
    assert f(g=tiled(N=96, K=384)) == _abi.ERR_SHAPE and f(dt=7) == _abi.ERR_SHAPE
    assert f(ws=None) == _abi.ERR_WORKSPACE and f(nb=need - 1) == _abi.ERR_WORKSPACE
    assert b"workspace" in lib.tpdq_last_error()
    assert f(ws=(1 << 28) + 8) == _abi.ERR_ALIGN
    assert lib.tpdq_mx_workspace_bytes(_abi.OP_MX_MLP, 0, ref_of(up), ref_of(down)) == 0
    assert lib.tpdq_mx_workspace_bytes(_abi.OP_MX_MLP, 4, ref_of(up), ref_of(up)) == 0
    assert lib.tpdq_mx_workspace_bytes(7, 4, ref_of(up), ref_of(down)) == 0


def test_binding_refuses_on_the_host():
    import torch
    import paper_2402_04925_amd as tpdq
    X = torch.zeros(4, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        tpdq.mx_quantize(X, tpdq.MX_FP8)                      # not on a GPU
    with pytest.raises(ValueError):
        tpdq.MxTensor.empty(4, 64, 3, "cpu")
    with pytest.raises(ValueError):
        tpdq.MxTensor.from_tensors(torch.zeros(4, 48, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 64, tpdq.MX_FP4)
    w = tpdq.MxTensor.empty(96, 1536, tpdq.MX_FP4, "cpu", tpdq.MX_TILED)
    with pytest.raises(ValueError):
        w.column_shard(0, 2)                                  # 48 rows: no whole tiles
    with pytest.raises(ValueError):
        w.row_shard(0, 2)                                     # 768 inputs: no whole chunks
    with pytest.raises(ValueError):
        w.column_shard(0, 5)                                  # 96 / 5
    with pytest.raises(ValueError):
        w.scales
    assert w.row_shard(1, 3).codes.shape == (3, 4 * 2048) and w.row_shard(1, 3).padded_scales.shape == (3, 512)
    with pytest.raises(ValueError):
        tpdq.mx_gemm(tpdq.MxTensor.empty(1, 1536, tpdq.MX_FP8, "cpu"), w, torch.float16)


@pytest.mark.parametrize("fmt,layout", [(_abi.MX_FP4, _abi.MX_ROWS), (_abi.MX_FP8, _abi.MX_ROWS), (_abi.MX_FP4, _abi.MX_TILED)])
def test_views_cut_short_are_no_tensor(fmt, layout):
    """The leading dimension of a cut view is the whole row's: a call would read past
    the last row's end."""
    import torch
    import paper_2402_04925_amd as tpdq
    q = tpdq.MxTensor.empty(64, 1024, fmt, "cpu", layout)
    c, s = q.codes, q.padded_scales
    make = lambda c, s, K: tpdq.MxTensor(c, s, 64, K, fmt, layout)
    half_c, half_s = c.shape[1] // 2, s.shape[1] // 2
    assert make(c[:, half_c:], s[:, half_s:], 512).K == 512
    assert make(c[:, 16:], s, 896).K == 896
    for bad in ((c[:, half_c:], s, 1024), (c, s[:, half_s:], 1024), (c[:, 16:], s, 1024), (c[:, half_c:], s[:, half_s:], 520)):
        with pytest.raises(ValueError):
            make(*bad)
    with pytest.raises(ValueError):
        tpdq.MxTensor(c, s, 64, 1024, 2, layout)
