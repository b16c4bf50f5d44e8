"""Every kernel that a microscaled product can be planned for, against float64: each tile
shape and row bucket, with and without K split over workgroups, in both element types,
quantized and gated. tests/test_mx_routes.py checks on the host that ROUTES reach them.

The references are float64 products on the GPU of the operands' values (mx_dequantize in
bfloat16 is exact for them and has tests of its own)."""
import numpy as np
import pytest

import paper_2402_04925_amd as tpdq
from tests import gpu_util as u
from tests import mx_ref as ref
from tests.test_gpu_mx import TINY, eps_half, sum_err, torch_dt

pytestmark = pytest.mark.gpu

FMTS = [tpdq.MX_FP4, tpdq.MX_FP8]
DTS = ["fp16", "bf16"]

# (M, N, K), no whole tile, step or chunk among them
ROUTES = [(1, 264, 272), (2, 4200, 264), (18, 272, 264), (18, 272, 24592), (18, 25304, 21568), (19, 4312, 264),
          (34, 4176, 272), (35, 264, 272), (37, 16944, 16528), (42, 4136, 2568), (66, 272, 1632), (66, 272, 3728),
          (143, 11240, 22464), (1339, 1576, 9752), (1366, 296, 7976), (1827, 272, 17856), (2144, 2000, 12080),
          (2721, 336, 20240), (2771, 680, 272), (2896, 2824, 1096), (3545, 3504, 264), (3688, 1072, 264)]


def activations(M, K, fmt, dev):
    """(MxTensor, float64 values)"""
    import torch
    g = torch.Generator(device=dev).manual_seed(M + K)
    x = torch.randn(M, K, generator=g, device=dev) * torch.exp(0.5 * torch.randn(K, generator=g, device=dev))
    q = tpdq.mx_quantize(x.to(torch.bfloat16), fmt)
    return q, tpdq.mx_dequantize(q, torch.bfloat16).double()


def weights(N, K, seed, dev, rows=None):
    """(MxTensor tiled, float64 values of all or some rows); products of K come out near 1."""
    import torch
    g = torch.Generator(device=dev).manual_seed(seed + N + K)
    nb = -(-K // 32)
    codes = torch.randint(0, 256, (N, nb * 16), generator=g, device=dev, dtype=torch.uint8)
    low = 127 - int(np.log2(K) / 2) - 3
    sb = torch.randint(low, low + 3, (N, nb), generator=g, device=dev, dtype=torch.uint8)
    q = tpdq.MxTensor.from_tensors(codes, sb, K, tpdq.MX_FP4)
    v = tpdq.mx_dequantize(q, torch.bfloat16)
    return tpdq.mx_pack(q), (v if rows is None else v[rows]).double()


class Product:
    """x w^T in float64; `most`, how far its fp32 sum may be off (as sum_bound in
    test_gpu_mx.py), and `rms`, its root mean square at most: of the fp32 chain's K / 128 + 40
    roundings of 2^-23 of a partial sum, as large as the whole; and with an fp8 operand of the
    up to 7 products in each 8 that lose less than 2^(E - 13) each, 2^E <= 2 max|x| max|w|,
    evenly spread (a third of the square) and with the products' signs."""

    def __init__(self, x, w, fmt):
        K = x.shape[1]
        self.parts = 12 if fmt == tpdq.MX_FP8 else 8  # check()
        t = lambda a: a.t().contiguous()
        self.want = x @ t(w)
        self.most = sum_err(K) * (x.abs() @ t(w.abs()))
        var = (K / 128 + 40) * 2.0 ** -46 * (x.square() @ t(w.square()))
        if fmt == tpdq.MX_FP8:
            x8, w8 = (a.abs().view(a.shape[0], -1, 8).amax(-1) for a in (x, w))
            self.most += 2.0 ** -9 * (x8 @ t(w8))
            var += 7 / 3 * 2.0 ** -24 * (x8.square() @ t(w8.square()))
        self.rms = var.sqrt()

    def check(self, y, dt):
        import torch
        err = (y.double() - self.want).abs()
        assert (err <= eps_half(dt) * self.want.abs() + self.most + TINY[dt]).all()
        # as a whole: a rounding is even over a step of the output's type (a twelfth of its square). Sums of
        # fp4 products are whole multiples of a power of two, m = 2^k points to a step: what is rounded off is
        # j / m of a step, j = -m/2 + 1 .. m/2, whose mean square is (1 + 2 / m^2) / 12, at most an eighth
        # (m = 2: 0 and 1/2). The mean over n outputs is uncertain by a few of 1 / sqrt(n).
        low, places = (-14, 10) if dt == "fp16" else (-126, 7)
        step = torch.exp2(torch.floor(torch.log2(self.want.abs().clamp(min=2.0 ** low))) - places)
        allowed = (step.square() / self.parts + self.rms.square()).mean()
        assert err.square().mean() <= (1.02 + 5 / np.sqrt(err.numel())) * allowed, (err.square().mean() / allowed).sqrt()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", ROUTES)
def test_product(fmt, dt, M, N, K):
    dev = u.torch_dev()
    q, x = activations(M, K, fmt, dev)
    w, wv = weights(N, K, 1, dev)
    Product(x, wv, fmt).check(tpdq.mx_gemm(q, w, torch_dt(dt)), dt)


def picks(cols, K, dev):
    """A weight whose outputs are the columns `cols` of its input."""
    import torch
    codes = torch.zeros(len(cols), -(-K // 32) * 16, dtype=torch.uint8, device=dev)
    c = torch.as_tensor(cols, device=dev)
    codes[torch.arange(len(cols), device=dev), c // 2] = torch.where(c % 2 == 0, 0x02, 0x20).to(torch.uint8)  # ones
    sb = torch.full((len(cols), -(-K // 32)), 127, dtype=torch.uint8, device=dev)
    return tpdq.mx_pack(tpdq.MxTensor.from_tensors(codes, sb, K, tpdq.MX_FP4))


def gated_product(gate, up):
    """silu(gate) * up with `most` and `rms`: |silu'| <= 1.1; the exponential, a division and two
    products in fp32 are within 2^-20."""
    import torch
    s = gate.want * torch.sigmoid(gate.want)
    y = Product.__new__(Product)
    y.want = s * up.want
    first = lambda d, dg: s.abs() * d + (1.1 * dg + 2.0 ** -20 * s.abs()) * (up.want.abs() + d)
    y.most, y.rms = first(up.most, gate.most), first(up.rms, gate.rms)
    return y


def check_quantized(v, y, fmt):
    """v [M][n], whole blocks of columns and a last one that may be cut: what y comes out as."""
    want, most, rms = (t.cpu().numpy() for t in (y.want, y.most, y.rms))
    n = want.shape[1]
    scale = lambda a: np.repeat(ref.scales(ref.quantize(a, fmt)[1]), 32, axis=1)[:, :n]
    hi, lo = scale(np.abs(want) + most), scale(np.maximum(np.abs(want) - most, 0))
    top = ref.table(fmt)[-1]
    near = np.abs(v - want) <= ref.half_step((np.abs(want) + most) / hi, fmt) * hi * (1 + 1e-12) + most
    full = [(np.abs(want) + most >= top * s) & (v == np.copysign(top * s, want)) for s in (hi, lo)]
    assert (near | full[0] | full[1]).all()
    # as a whole: a sum off by e rounds the other way in e / step of the cases, of which the mean of
    # |e| is at most rms. Blocks whose scale is in doubt are left out (four rms).
    sure = scale(np.abs(want) + 4 * rms) == scale(np.maximum(np.abs(want) - 4 * rms, 0))
    step = 2 * ref.half_step(want / hi, fmt) * hi
    expected = (rms / step)[sure].sum()
    got = (v != ref.values(*ref.quantize(want, fmt), fmt).astype(np.float16))[sure].sum()
    assert got <= 1.1 * expected + 6 * np.sqrt(expected) + 5, (got, expected, sure.sum())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", ROUTES)
def test_first_product_of_the_mlp(gated, fmt, M, N, K):
    """Y1 as codes: w_down hands 16 blocks of its columns through (a product with ones and zeros
    is exact, and what fp16 holds of a code times its scale)."""
    import torch
    dev = u.torch_dev()
    blocks = -(-N // 32)
    some = np.unique(np.append(np.random.default_rng(N).integers(0, blocks, 14), [0, blocks - 1]))
    cols = np.concatenate([np.arange(32 * b, min(32 * b + 32, N)) for b in some])
    q, x = activations(M, K, fmt, dev)
    w, wv = weights(N, K, 1, dev, cols)
    y, gate = Product(x, wv, fmt), None
    if gated:
        gate, gv = weights(N, K, 2, dev, cols)
        y = gated_product(Product(x, gv, fmt), y)
    v = tpdq.mx_mlp_shard(q, w, picks(cols, N, dev), torch.float16, w_gate=gate)
    check_quantized(v.double().cpu().numpy(), y, fmt)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,K,N1,N2", [(1, 272, 264, 520), (16, 1160, 520, 1000), (64, 520, 1160, 72), (70, 384, 1000, 264),
                                       (300, 512, 648, 1096), (700, 1544, 1096, 392)])
def test_second_product_of_the_mlp(fmt, dt, M, K, N1, N2, gated):
    """Y2 of the codes that Y1 came out as (read through ones and zeros), in both types."""
    import torch
    dev = u.torch_dev()
    q, _ = activations(M, K, fmt, dev)
    w, _ = weights(N1, K, 1, dev)
    gate = weights(N1, K, 2, dev)[0] if gated else None
    down, dv = weights(N2, N1, 3, dev)
    y1 = tpdq.mx_mlp_shard(q, w, picks(np.arange(N1), N1, dev), torch.bfloat16, w_gate=gate).double()
    Product(y1, dv, fmt).check(tpdq.mx_mlp_shard(q, w, down, torch_dt(dt), w_gate=gate), dt)
