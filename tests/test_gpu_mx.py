"""The microscaled operators on the GPU against tests/mx_ref.py (float64)."""
import numpy as np
import pytest

import paper_2402_04925_amd as tpdq
from tests import gpu_util as u
from tests import mx_ref as ref

pytestmark = pytest.mark.gpu

FMTS = [tpdq.MX_FP4, tpdq.MX_FP8]
DTS = ["fp16", "bf16"]


def torch_dt(dt):
    import torch
    return torch.float16 if dt == "fp16" else torch.bfloat16


def f64(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def eps_half(dt):
    """One rounding to the type, relative."""
    return 2.0 ** -11 if dt == "fp16" else 2.0 ** -8


TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half the smallest subnormal step


def acts(R, K, seed, dev, dt, ld=None, outliers=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, K if ld is None else ld, generator=g)
    if outliers:
        x *= torch.exp(torch.randn(x.shape[1], generator=g))
    return x.to(torch_dt(dt)).to(dev)[:, :K]


def weight(N, K, seed, dev):
    """(MxTensor tiled, float64 values)"""
    import torch
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    sb = rng.integers(118, 122, (N, -(-K // 32))).astype(np.uint8)
    q = tpdq.MxTensor.from_tensors(torch.from_numpy(ref.pack_bytes(codes, ref.FP4)).to(dev),
                                   torch.from_numpy(sb).to(dev), K, tpdq.MX_FP4)
    return tpdq.mx_pack(q), ref.values(codes, sb, ref.FP4)


def quantized(M, K, fmt, seed, dev):
    """(MxTensor rows, float64 values) of random activations"""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((M, K)) * np.exp(rng.standard_normal(K))
    codes, sb = ref.quantize(x, fmt)
    b = torch.from_numpy(ref.pack_bytes(codes, fmt)).to(dev)
    if fmt == tpdq.MX_FP8:
        b = b.view(torch.float8_e4m3fn)
    return tpdq.MxTensor.from_tensors(b, torch.from_numpy(sb).to(dev), K, fmt), ref.values(codes, sb, fmt)


def raw(q):
    """(codes one each, scale bytes, all code bytes, all scale bytes) of an MX_ROWS tensor"""
    import torch
    c, s = q.codes.view(torch.uint8).cpu().numpy(), q.padded_scales.view(torch.uint8).cpu().numpy()
    return ref.unpack_bytes(c, q.K, q.fmt), s[:, :-(-q.K // 32)], c, s


def check_padding(q):
    _, _, c, s = raw(q)
    assert (c[:, q.K // 2 if q.fmt == tpdq.MX_FP4 else q.K:] == 0).all()
    assert (s[:, -(-q.K // 32):] == 0).all()


# ---- quantize, dequantize, pack ------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("R,K", [(1, 8), (1, 24), (3, 32), (2, 40), (5, 504), (4, 512), (7, 520), (33, 5000), (1, 8192)])
def test_quantize(fmt, dt, R, K):
    dev = u.torch_dev()
    x = acts(R, K, R * 1000 + K, dev, dt, ld=K + 8)
    if K > 64:
        x[0, 32:64] = 0
    q = tpdq.mx_quantize(x, fmt)
    codes, sb = ref.quantize(f64(x), fmt)
    got = raw(q)
    np.testing.assert_array_equal(got[1], sb)
    np.testing.assert_array_equal(got[0], codes)
    check_padding(q)
    np.testing.assert_array_equal(q.scales.float().double().cpu().numpy(), ref.scales(sb))
    # and back: one rounding of an exact product
    v = ref.values(codes, sb, fmt)
    back = f64(tpdq.mx_dequantize(q, x.dtype))
    assert (np.abs(back - v) <= eps_half(dt) * np.abs(v) + TINY[dt]).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", DTS)
def test_quantize_every_16_bit_value(fmt, dt):
    """Every finite bit pattern beside an anchor at its own power of two and beside
    one 2^6 above, and in a block of itself: all ties, subnormals and saturations."""
    import torch
    dev = u.torch_dev()
    b = np.arange(65536, dtype=np.uint16)
    x = torch.from_numpy(b.view(np.int16).copy()).view(torch_dt(dt)).double().numpy()
    x = x[np.isfinite(x)]
    most = 65504.0 if dt == "fp16" else 2.0 ** 127
    rows = np.zeros((len(x), 32))
    rows[:, 0] = x
    rows[::3, 1] = np.minimum(2.0 ** np.floor(np.log2(np.maximum(np.abs(x[::3]), 1e-40))), most)
    rows[1::3, 1] = np.minimum(np.maximum(np.abs(x[1::3]), 1e-40) * 64, most)
    t = torch.from_numpy(rows).to(torch_dt(dt)).to(dev)
    q = tpdq.mx_quantize(t, fmt)
    codes, sb = ref.quantize(f64(t), fmt)
    got = raw(q)
    np.testing.assert_array_equal(got[1], sb)
    np.testing.assert_array_equal(got[0], codes)


@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_not_finite(fmt):
    import torch
    dev = u.torch_dev()
    x = torch.ones(4, 96, dtype=torch.bfloat16, device=dev)
    x[0, 5], x[1, 33], x[2, 95], x[3, :] = float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min
    q = tpdq.mx_quantize(x, fmt)
    codes, sb = ref.quantize(f64(x), fmt)
    assert (sb == 255).sum() == 3
    np.testing.assert_array_equal(raw(q)[1], sb)
    np.testing.assert_array_equal(raw(q)[0], codes)
    back = tpdq.mx_dequantize(q, torch.bfloat16)
    assert torch.isnan(back).sum() == 96 and torch.isfinite(back[3]).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_dequantize_every_code_and_scale(fmt):
    import torch
    dev = u.torch_dev()
    n = 16 if fmt == tpdq.MX_FP4 else 256
    K = max(32, n)
    codes = np.tile(np.arange(K) % n, (256, 1)).astype(np.uint8)
    sb = np.repeat(np.arange(256, dtype=np.uint8)[:, None], K // 32, axis=1)
    b = torch.from_numpy(ref.pack_bytes(codes, fmt)).to(dev)
    q = tpdq.MxTensor.from_tensors(b.view(torch.float8_e4m3fn) if fmt == tpdq.MX_FP8 else b, torch.from_numpy(sb).to(dev), K, fmt)
    got = f64(tpdq.mx_dequantize(q, torch.bfloat16))
    v = ref.values(codes, sb, fmt)
    most = float(torch.finfo(torch.bfloat16).max)
    fin = np.abs(v) <= most
    assert (np.isnan(got) == np.isnan(v)).all()
    assert (np.abs(got - v)[fin] <= eps_half("bf16") * np.abs(v)[fin] + TINY["bf16"]).all()
    assert np.isinf(got[np.abs(v) >= 2.0 ** 128]).all()


@pytest.mark.parametrize("N,K", [(8, 8), (32, 128), (40, 136), (64, 512), (72, 1000)])
def test_pack(N, K):
    import torch
    dev = u.torch_dev()
    rng = np.random.default_rng(N + K)
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    sb = rng.integers(0, 255, (N, -(-K // 32))).astype(np.uint8)
    q = tpdq.MxTensor.from_tensors(torch.from_numpy(ref.pack_bytes(codes, ref.FP4)).to(dev), torch.from_numpy(sb).to(dev),
                                   K, tpdq.MX_FP4)
    q.codes[:, K // 2:] = 0x77  # what lies past K does not reach the tiles
    w = tpdq.mx_pack(q)
    c, s = ref.tiled(codes, sb)
    np.testing.assert_array_equal(w.codes.cpu().numpy(), c)
    np.testing.assert_array_equal(w.padded_scales.view(torch.uint8).cpu().numpy(), s)


def test_past_32_bits():
    """More than 2^32 elements: the last rows of a quantization, its inverse and a norm."""
    import torch
    dev = u.torch_dev()
    R, K = 70000, 65536
    x = torch.zeros(R, K, dtype=torch.bfloat16, device=dev)
    x[-3:] = acts(3, K, 5, dev, "bf16")
    q = tpdq.mx_quantize(x, tpdq.MX_FP8)
    tail = tpdq.mx_quantize(x[-3:], tpdq.MX_FP8)
    assert torch.equal(q.codes[-3:].view(torch.uint8), tail.codes.view(torch.uint8))
    assert torch.equal(q.padded_scales[-3:].view(torch.uint8), tail.padded_scales.view(torch.uint8))
    w = torch.ones(K, dtype=torch.bfloat16, device=dev)
    y, _ = tpdq.rmsnorm(x, w, 1e-5, out=x)  # a row is read before it is written
    want, _ = tpdq.rmsnorm(acts(3, K, 5, dev, "bf16"), w, 1e-5)
    assert torch.equal(y[-3:], want)
    back = tpdq.mx_dequantize(q, torch.bfloat16, out=x)
    assert torch.equal(back[-3:], tpdq.mx_dequantize(tail, torch.bfloat16)) and not back[:3].any()


# ---- norm ----------------------------------------------------------------

# The sum of squares: at most 64 terms in a lane, 6 + 16 levels above, each 2^-24;
# the root, the division and three products are a few more: 100 x 2^-24 < 2^-17.
NORM_ERR = 2.0 ** -17


@pytest.mark.parametrize("fmt", [None] + FMTS)
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("M,K", [(1, 8), (3, 40), (2, 1000), (5, 4096), (4, 6144), (1, 8192), (2, 16392), (2, 65536)])
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm(fmt, dt, M, K, residual):
    import torch
    dev = u.torch_dev()
    x = acts(M, K, M + K, dev, dt, ld=K + 16)
    res = acts(M, K, M + K + 1, dev, dt, ld=K + 8) if residual else None
    w = (1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))).to(torch_dt(dt)).to(dev)
    y, h = tpdq.rmsnorm(x, w, 1e-5, residual=res, fmt=fmt)
    want_h = x if res is None else (x.float() + res.float()).to(x.dtype)
    assert torch.equal(h, want_h)
    want = ref.rmsnorm(f64(want_h), f64(w), 1e-5)
    if fmt is None:
        assert (np.abs(f64(y) - want) <= (eps_half(dt) + NORM_ERR) * np.abs(want) + TINY[dt]).all()
        return
    check_padding(y)
    codes, sb, _, _ = raw(y)
    check_quantized(want, codes, sb, fmt, NORM_ERR)


def check_quantized(want, codes, sb, fmt, err):
    """codes and scales are those of numbers within a relative err of `want`."""
    s = np.repeat(ref.scales(sb), 32, axis=1)[:, :want.shape[1]]
    lo, hi = (ref.quantize(want * f, fmt)[1].astype(int) for f in (1 - 2 * err, 1 + 2 * err))
    assert ((sb >= lo) & (sb <= hi)).all()
    v, a = ref.elements(codes, fmt), want / s
    most = ref.table(fmt)[-1]
    near = np.abs(v - a) <= ref.half_step(a, fmt) * (1 + 1e-12) + err * np.abs(a)
    assert (near | ((np.abs(a) * (1 + err) >= most) & (v == np.copysign(most, a)))).all()


def test_rmsnorm_in_place_and_strided_outputs():
    import torch
    dev = u.torch_dev()
    M, K = 6, 1000
    x, res = acts(M, K, 1, dev, "bf16"), acts(M, K, 2, dev, "bf16")
    w = torch.ones(K, dtype=torch.bfloat16, device=dev)
    y, h = tpdq.rmsnorm(x, w, 1e-6, residual=res)
    wide = torch.full((M + 2, K + 24), 7.0, dtype=torch.bfloat16, device=dev)
    mine = res.clone()
    y2, h2 = tpdq.rmsnorm(x, w, 1e-6, residual=mine, residual_out=mine, out=wide[1:M + 1, 8:K + 8])
    assert h2 is mine and torch.equal(mine, h) and torch.equal(y2, y)
    wide[1:M + 1, 8:K + 8] = 7.0
    assert (wide == 7.0).all()  # nothing beside the output was written


def test_rmsnorm_rows_that_are_not_finite_or_zero():
    import torch
    dev = u.torch_dev()
    K = 520
    x = acts(4, K, 3, dev, "bf16")
    w = torch.ones(K, dtype=torch.bfloat16, device=dev)
    x[0, 7], x[1, 9], x[2, :] = float("nan"), float("inf"), 0
    y, _ = tpdq.rmsnorm(x, w, 1e-5)
    q, _ = tpdq.rmsnorm(x, w, 1e-5, fmt=tpdq.MX_FP8)
    v = tpdq.mx_dequantize(q, torch.bfloat16)
    assert torch.isnan(y[0]).all() and torch.isnan(v[0]).all()
    assert torch.isnan(y[1, 9]) and (torch.cat([y[1, :9], y[1, 10:]]) == 0).all()
    assert torch.isnan(v[1, :32]).all() and (v[1, 32:] == 0).all()
    assert (y[2] == 0).all() and (v[2] == 0).all() and torch.isfinite(y[3]).all()
    check_padding(q)


# ---- product -------------------------------------------------------------

def sum_err(K):
    """fp32 sums of exact products: a chain of K / 128 instructions, each adding its
    128 products with a few roundings or truncations (2^-23 each), then up to 16
    partial sums; relative to the sum of magnitudes."""
    return (K / 128 + 40) * 2.0 ** -23


def eights(x):
    """The largest magnitude of each 8 consecutive elements."""
    K = x.shape[1]
    full = np.zeros((x.shape[0], -(-K // 8) * 8))
    full[:, :K] = np.abs(x)
    return full.reshape(x.shape[0], -(-K // 8), 8).max(-1)


def sum_bound(x, w, fmt):
    """How far a sum of products may be off. With an fp8 operand the matrix
    instruction aligns each 8 consecutive products to the largest of their exponent
    sums E and drops what lies below 2^(E - 13) (seen by adding 2^-j to 256: lost from
    j = 6 on, for the 7 elements beside it and no others). An operand of exponent e is
    at least 2^e, but for an fp4 0.5, which counts as e = 0 (subnormal fp8 products are
    multiples of 2^-10 and lose nothing at their E <= -4): 2^E <= 2 max|x| max|w|, and 7
    products lose 7 x 2^-13 x 2 < 2^-9 of that."""
    b = sum_err(x.shape[1]) * (np.abs(x) @ np.abs(w).T)
    return b + 2.0 ** -9 * (eights(x) @ eights(w).T) if fmt == tpdq.MX_FP8 else b


def check_product(y, x, w, dt, fmt):
    want = x @ w.T
    err = np.abs(f64(y) - want)
    bound = sum_bound(x, w, fmt)
    assert (err <= eps_half(dt) * np.abs(want) + bound + TINY[dt]).all(), (err / bound).max()


SHAPES = [(1, 8, 8), (1, 32, 32), (3, 40, 136), (16, 64, 512), (17, 96, 520), (33, 104, 1000), (64, 72, 5000),
          (5, 3464, 1024), (2, 64, 16384), (65, 256, 256), (77, 520, 1160), (128, 264, 640), (200, 1000, 384), (257, 512, 2048),
          (300, 136, 136)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(fmt, dt, M, N, K):
    import torch
    dev = u.torch_dev()
    q, x = quantized(M, K, fmt, M + N + K, dev)
    w, wv = weight(N, K, N + K, dev)
    wide = torch.full((M + 2, N + 16), 3.0, dtype=torch_dt(dt), device=dev)
    y = tpdq.mx_gemm(q, w, torch_dt(dt), out=wide[1:M + 1, 8:N + 8])
    check_product(y, x, wv, dt, fmt)
    assert torch.equal(y, tpdq.mx_gemm(q, w, torch_dt(dt)))  # the same bits again
    wide[1:M + 1, 8:N + 8] = 3.0
    assert (wide == 3.0).all()


# sizes where other tiles and splits are chosen: real layers, sampled
LARGE = [(1, 3584, 8192), (16, 8192, 3584), (24, 6144, 6144), (64, 28672, 8192), (100, 8192, 8192), (256, 3584, 8192),
         (512, 6144, 6144), (1000, 3584, 8192), (2048, 8192, 3584), (70, 512, 28672)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", LARGE)
def test_product_of_real_layers(fmt, M, N, K):
    import torch
    dev = u.torch_dev()
    g = torch.Generator(device=dev).manual_seed(M + N + K)
    q = tpdq.mx_quantize(acts(M, K, M + K, dev, "bf16"), fmt)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device=dev, dtype=torch.uint8)
    sb = torch.randint(118, 122, (N, K // 32), generator=g, device=dev, dtype=torch.uint8)
    wq = tpdq.MxTensor.from_tensors(codes, sb, K, tpdq.MX_FP4)
    y = tpdq.mx_gemm(q, tpdq.mx_pack(wq), torch.bfloat16)
    x = tpdq.mx_dequantize(q, torch.bfloat16).double()  # exact: 4 significant bits, scales within the type's range
    w = tpdq.mx_dequantize(wq, torch.bfloat16).double()
    want, mag = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
    bound = sum_err(K) * mag
    if fmt == tpdq.MX_FP8:  # sum_bound()
        bound += 2.0 ** -9 * (x.abs().view(M, -1, 8).amax(-1) @ w.abs().view(N, -1, 8).amax(-1).t().contiguous())
    err = (y.double() - want).abs()
    assert (err <= eps_half("bf16") * want.abs() + bound).all(), (err / bound).max()
    # and as a whole no more than the output's rounding
    assert err.square().mean().sqrt() <= eps_half("bf16") * want.square().mean().sqrt()


# ragged sizes (K and N in no whole block, step, chunk or tile) that reach every tile
# shape, in 16 bits, quantized and gated (tests/test_mx_ref.py checks that they do)
TILES = [(1155, 8984, 328), (1421, 2976, 456), (223, 8248, 584), (1639, 4632, 1160), (2040, 8184, 1032), (1526, 5400, 904),
         (43, 40, 2680), (40, 14344, 1160), (30, 4360, 1096), (100, 360, 5000),
         (101, 968, 2632), (149, 240, 3088), (1027, 136, 10072), (100, 1016, 1176), (593, 6480, 192)]


def some_rows(M, seed):
    """Edges of the row tiles and random rows."""
    rng = np.random.default_rng(seed)
    edges = [r for t in (16, 64, 128) for r in (0, t - 1, t, M // t * t - 1, M // t * t, M - 1)]
    return np.unique(np.clip(edges + rng.integers(0, M, 24).tolist(), 0, M - 1))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", TILES)
def test_product_tiles(fmt, M, N, K):
    dev = u.torch_dev()
    q, x = quantized(M, K, fmt, M + N + K, dev)
    w, wv = weight(N, K, N + K, dev)
    rows = some_rows(M, N)
    check_product(tpdq.mx_gemm(q, w, torch_dt("bf16"))[rows], x[rows], wv, "bf16", fmt)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", TILES)
def test_mlp_tiles(gated, fmt, M, N, K):
    dev = u.torch_dev()
    N2 = 72
    q, x = quantized(M, K, fmt, M + N + K, dev)
    (wu, wuv), (wd, wdv) = weight(N, K, 1, dev), weight(N2, N, 2, dev)
    wg, wgv = weight(N, K, 3, dev) if gated else (None, None)
    rows = some_rows(M, N)
    y = tpdq.mx_mlp_shard(q, wu, wd, torch_dt("bf16"), w_gate=wg)[rows]
    want, bound = mlp_want(x[rows], wuv, wdv, wgv, fmt)
    err = np.abs(f64(y) - want)
    assert (err <= eps_half("bf16") * np.abs(want) + bound).all(), (err / bound).max()
    assert np.sqrt((err * err).mean()) <= 2.0 ** -6 * np.sqrt((want * want).mean())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M", [1, 20, 64, 130, 300])
def test_product_not_finite(fmt, M):
    """A NaN scale in one row of X, one of w: that row and that column alone."""
    import torch
    dev = u.torch_dev()
    N, K = 96, 1096
    q, x = quantized(M, K, fmt, 4, dev)
    q.padded_scales.view(torch.uint8)[M // 2, 3] = 255
    w0, wv = weight(N, K, 5, dev)
    w = tpdq.MxTensor(w0.codes.clone(), w0.padded_scales.clone(), N, K, w0.fmt, w0.layout)
    w.padded_scales.view(torch.uint8)[1, 512 + 8 * 5 + 1] = 255  # tile 1, chunk 1, lane 5, operand 0, step 1: row 32 + 8 + 1
    y = f64(tpdq.mx_gemm(q, w, torch.bfloat16))
    bad = np.zeros((M, N), bool)
    bad[M // 2], bad[:, 41] = True, True
    assert (np.isnan(y) == bad).all()
    clean = np.delete(np.delete(y, M // 2, 0), 41, 1)
    check_product(torch.from_numpy(clean), np.delete(x, M // 2, 0), np.delete(wv, 41, 0), "bf16", fmt)


def test_product_scales_at_both_ends():
    """The smallest and largest scales multiply exactly where the product is in range."""
    import torch
    dev = u.torch_dev()
    for a, b in ((0, 254), (1, 250), (127, 127), (254, 0), (30, 200)):
        c = torch.full((16, 64), 0x22, dtype=torch.uint8, device=dev)  # ones
        q = tpdq.MxTensor.from_tensors(c, torch.full((16, 4), a, dtype=torch.uint8, device=dev), 128, tpdq.MX_FP4)
        w = tpdq.MxTensor.from_tensors(torch.cat([c, c]), torch.full((32, 4), b, dtype=torch.uint8, device=dev), 128, tpdq.MX_FP4)
        y = f64(tpdq.mx_gemm(q, tpdq.mx_pack(w), torch.bfloat16))
        assert (y == 128 * 2.0 ** (a + b - 254)).all(), (a, b, y[0, 0])


# ---- MLP -----------------------------------------------------------------

def mlp_want(x, wu, wd, wg, fmt):
    """Y2 in float64, and how far its sum may be off, codes of Y1 included that the
    kernel's sums may round the other way. fp32 silu (the exponential within 2^-21, a
    division and two products) and sums: Y1 is known to d."""
    up = x @ wu.T
    d = sum_bound(x, wu, fmt)
    y1 = up
    if wg is not None:
        gate = x @ wg.T
        dg = sum_bound(x, wg, fmt)
        y1 = ref.silu(gate) * up
        # |silu'| <= 1.1
        d = np.abs(ref.silu(gate)) * d + (1.1 * dg + 2.0 ** -20 * np.abs(ref.silu(gate))) * (np.abs(up) + d)
    vals = []
    for y in (y1, y1 - d, y1 + d):
        vals.append(ref.values(*ref.quantize(y, fmt), fmt))
    doubt = np.maximum(np.abs(vals[1] - vals[0]), np.abs(vals[2] - vals[0]))
    # a scale that may be the other power of two: every element of the block to half a step of both
    top = lambda y: ref.quantize(y, fmt)[1]
    up1 = np.abs(y1) + d
    lo1 = np.maximum(np.abs(y1) - d, 0)
    unsure = top(up1) != top(lo1)
    blk = np.repeat(unsure, 32, axis=1)[:, :y1.shape[1]]
    s = np.repeat(ref.scales(top(up1)), 32, axis=1)[:, :y1.shape[1]]
    # halved scale: up to a step of rounding and a quarter of saturation (fp4: 8 -> 6)
    doubt = np.where(blk, np.maximum(doubt, s * 2 * ref.half_step(y1 / s, fmt) + 0.25 * np.abs(y1)), doubt)
    return vals[0] @ wd.T, 1.01 * doubt @ np.abs(wd).T + sum_bound(np.abs(vals[0]) + doubt, wd, fmt)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,K1,N1,N2", [(1, 128, 32, 8), (3, 520, 136, 40), (16, 1024, 256, 520), (20, 384, 1000, 64),
                                       (70, 256, 520, 264), (130, 1160, 384, 96), (300, 512, 640, 512)])
def test_mlp(gated, fmt, M, K1, N1, N2):
    import torch
    dev = u.torch_dev()
    q, x = quantized(M, K1, fmt, M + K1, dev)
    (wu, wuv), (wd, wdv) = weight(N1, K1, 1, dev), weight(N2, N1, 2, dev)
    wg, wgv = weight(N1, K1, 3, dev) if gated else (None, None)
    y = tpdq.mx_mlp_shard(q, wu, wd, torch.bfloat16, w_gate=wg)
    want, bound = mlp_want(x, wuv, wdv, wgv, fmt)
    err = np.abs(f64(y) - want)
    assert (err <= eps_half("bf16") * np.abs(want) + bound).all(), (err / bound).max()
    # the bound counts every code in doubt at once; as a whole the result is much nearer
    assert np.sqrt((err * err).mean()) <= 2.0 ** -6 * np.sqrt((want * want).mean())
    assert torch.equal(y, tpdq.mx_mlp_shard(q, wu, wd, torch.bfloat16, w_gate=wg, workspace=tpdq.Workspace(dev)))


@pytest.mark.parametrize("fmt", FMTS)
def test_layer_as_used_and_over_ranks(fmt):
    """Norm with the residual -> gated MLP share of two ranks -> their sum into the
    next norm; each rank's share against float64, and the sum against one rank's."""
    import torch
    dev = u.torch_dev()
    M, K, N1 = 9, 1024, 1024
    x, res = acts(M, K, 1, dev, "bf16"), acts(M, K, 2, dev, "bf16")
    nw = torch.ones(K, dtype=torch.bfloat16, device=dev)
    q, h = tpdq.rmsnorm(x, nw, 1e-5, residual=res, fmt=fmt)
    xv = ref.values(raw(q)[0], raw(q)[1], fmt)
    (wu, wuv), (wg, wgv), (wd, wdv) = (weight(*s, i, dev) for i, s in enumerate([(N1, K), (N1, K), (K, N1)]))
    total, wants, bounds = 0, 0, 0
    for r in range(2):
        part = tpdq.mx_mlp_shard(q, wu.column_shard(r, 2), wd.row_shard(r, 2), torch.bfloat16, w_gate=wg.column_shard(r, 2))
        c = slice(r * N1 // 2, (r + 1) * N1 // 2)
        want, bound = mlp_want(xv, wuv[c], wdv[:, c], wgv[c], fmt)
        bound += eps_half("bf16") * np.abs(want)
        assert (np.abs(f64(part) - want) <= bound).all()
        total, wants, bounds = total + part.float(), wants + want, bounds + bound
    # the ranks' shares add up to the whole MLP
    want, bound = mlp_want(xv, wuv, wdv, wgv, fmt)
    assert np.abs(wants - want).max() <= 1e-9 * np.abs(want).max()
    assert (np.abs(f64(total) - want) <= bounds + 2.0 ** -23 * np.abs(want)).all()
    whole = tpdq.mx_mlp_shard(q, wu, wd, torch.bfloat16, w_gate=wg)
    assert (np.abs(f64(whole) - want) <= eps_half("bf16") * np.abs(want) + bound).all()
    y, h2 = tpdq.rmsnorm(total.to(torch.bfloat16), nw, 1e-5, residual=h, residual_out=h)
    assert h2 is h and torch.isfinite(y).all()


def test_norm_feeds_the_w4a16_shard():
    """The norm's 16-bit output through the ordered W4A16 MLP share."""
    import torch
    from oracle import tpdq_oracle as o
    from paper_2402_04925_amd import inputs
    dev = u.torch_dev()
    L1, L2 = inputs.make_custom(256, 512, 256, 32, seed=3)
    d1, d2 = u.layer_to_dev(L1, dev), u.layer_to_dev(L2, dev)
    P1, _, P2, _, w1, w2 = tpdq.reorder(d1, d2)
    x, res = acts(5, 256, 1, dev, "fp16", outliers=False), acts(5, 256, 2, dev, "fp16", outliers=False)
    y, h = tpdq.rmsnorm(x, torch.ones(256, dtype=torch.float16, device=dev), 1e-5, residual=res)
    _, y2 = tpdq.mlp_shard(y, w1, w2, tpdq.PATH_ORDERED, P1=P1)
    l1, l2 = ((L.qweight, L.scales, L.qzeros, L.g_idx) for L in (L1, L2))
    _, e2 = o.mlp_rank_from_global(u.np_of(y), l1, l2, 0, 1, True, P2=u.np_of(P2))
    assert o.rel_err(u.np_of(y2), e2) <= u.TOL_FP16


@pytest.mark.parametrize("M", [1, 16, 80, 300])
def test_captured_and_replayed(M):
    """The chain in a HIP graph, replayed with new inputs between eager calls, on
    a stream of its own; two graphs of the same tensors in turn."""
    import torch
    dev = u.torch_dev()
    K, N1 = 1024, 1056
    x, res = acts(M, K, 1, dev, "bf16"), acts(M, K, 2, dev, "bf16")
    nw = torch.ones(K, dtype=torch.bfloat16, device=dev)
    (wu, _), (wg, _), (wd, _) = (weight(*s, i, dev) for i, s in enumerate([(N1, K), (N1, K), (K, N1)]))

    def chain():
        q, h = tpdq.rmsnorm(x, nw, 1e-5, residual=res, fmt=tpdq.MX_FP8)
        y = tpdq.mx_mlp_shard(q, wu, wd, torch.bfloat16, w_gate=wg)
        z = tpdq.mx_gemm(tpdq.mx_quantize(y, tpdq.MX_FP4), wu, torch.bfloat16)
        return h, y, z

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    side.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(chain())
        graphs.append(g)
    for i in range(4):
        x.copy_(acts(M, K, 10 + i, dev, "bf16"))
        want = chain()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[i % 2].replay()
            graphs[1 - i % 2].replay()
        side.synchronize()
        for out in outs:
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls on two streams share nothing."""
    import torch
    dev = u.torch_dev()
    M, K, N1 = 64, 2048, 2048
    (wu, _), (wd, _) = weight(N1, K, 1, dev), weight(K, N1, 2, dev)
    qs = [quantized(M, K, tpdq.MX_FP8, i, dev)[0] for i in range(2)]
    want = [tpdq.mx_mlp_shard(q, wu, wd, torch.float16) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(tpdq.mx_mlp_shard(qs[i], wu, wd, torch.float16))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_one_row_of_whatever_stride():
    """torch keeps any stride for an axis of one: a row of a wider buffer, a turned column."""
    import torch
    dev = u.torch_dev()
    K, N = 520, 72
    x = acts(1, K, 1, dev, "bf16")
    nw = torch.ones(K, dtype=torch.bfloat16, device=dev)
    w, _ = weight(N, K, 2, dev)
    q = tpdq.mx_quantize(x, tpdq.MX_FP8)
    y, h = tpdq.rmsnorm(x, nw, 1e-5, residual=x)
    for ld in (1, 3, K + 4):
        turned = lambda n: torch.empty(max(n, ld), dtype=torch.bfloat16, device=dev).as_strided((1, n), (ld, 1))
        xt, out = turned(K), turned(N)
        xt.copy_(x)
        qt = tpdq.mx_quantize(xt, tpdq.MX_FP8)
        assert torch.equal(qt.codes.view(torch.uint8), q.codes.view(torch.uint8))
        assert torch.equal(tpdq.mx_dequantize(q, torch.bfloat16, out=turned(K)), tpdq.mx_dequantize(q, torch.bfloat16))
        yt, ht = tpdq.rmsnorm(xt, nw, 1e-5, residual=xt, residual_out=turned(K), out=turned(K))
        assert torch.equal(yt, y) and torch.equal(ht, h)
        assert torch.equal(tpdq.mx_gemm(q, w, torch.bfloat16, out=out), tpdq.mx_gemm(q, w, torch.bfloat16))


def test_binding_refuses():
    import torch
    dev = u.torch_dev()
    x = acts(4, 256, 1, dev, "fp16")
    q, _ = quantized(4, 256, tpdq.MX_FP8, 1, dev)
    w, _ = weight(64, 256, 2, dev)
    nw = torch.ones(256, dtype=torch.float16, device=dev)
    with pytest.raises(ValueError):
        tpdq.mx_quantize(x.t(), tpdq.MX_FP8)
    with pytest.raises(TypeError):
        tpdq.mx_quantize(x.float(), tpdq.MX_FP8)
    with pytest.raises(tpdq.TpdqError):
        tpdq.mx_quantize(x[:, 4:252], tpdq.MX_FP8)                     # 8-byte alignment
    with pytest.raises(tpdq.TpdqError):
        tpdq.mx_quantize(x[:, :100], tpdq.MX_FP8)                      # K % 8
    with pytest.raises(tpdq.TpdqError):
        tpdq.mx_quantize(x[:0], tpdq.MX_FP8)                           # no rows
    with pytest.raises(ValueError):
        tpdq.mx_quantize(x, tpdq.MX_FP8, out=tpdq.MxTensor.empty(4, 256, tpdq.MX_FP4, dev))
    with pytest.raises(tpdq.TpdqError):
        tpdq.mx_gemm(q, tpdq.MxTensor.empty(64, 256, tpdq.MX_FP4, dev), torch.float16)   # not packed
    with pytest.raises(tpdq.TpdqError):
        tpdq.mx_gemm(q, weight(64, 512, 3, dev)[0], torch.float16)
    with pytest.raises(TypeError):
        tpdq.mx_gemm(q, w, torch.float32)
    with pytest.raises(ValueError):
        tpdq.mx_gemm(q, w, torch.float16, out=torch.empty(4, 56, dtype=torch.float16, device=dev))
    with pytest.raises(TypeError):
        tpdq.rmsnorm(x, nw.bfloat16(), 1e-5)
    with pytest.raises(ValueError):
        tpdq.rmsnorm(x, nw[:128], 1e-5)
    with pytest.raises(ValueError):
        tpdq.rmsnorm(x, nw, 1e-5, residual_out=x)
    with pytest.raises(tpdq.TpdqError):
        tpdq.rmsnorm(x, nw, -1.0)
    with pytest.raises(ValueError):
        tpdq.mx_mlp_shard(q, w, w, torch.float16)                       # 64 outputs, 256 inputs
    with pytest.raises(TypeError):
        tpdq.mx_gemm(x, w, torch.float16)
    with pytest.raises(AttributeError):
        w.codes = w.codes
    d, _ = weight(64, 64, 3, dev)
    with pytest.raises(ValueError):
        tpdq.mx_mlp_shard(q, w, d, torch.float16, out=torch.empty(4, 128, dtype=torch.float16, device=dev)[:, :64])
