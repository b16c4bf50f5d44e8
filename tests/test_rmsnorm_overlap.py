"""tpdq_rmsnorm and memory that its arguments share: which calls are refused (fake
device pointers, no GPU), and that those it takes give the same bits (GPU)."""
import ctypes
import os

import pytest

from paper_2402_04925_amd import _abi

needs_no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake device pointers only where no GPU exists")

if not os.path.exists(_abi.LIB_PATH):
    from paper_2402_04925_amd import build
    build.build()

K, M = 256, 4
ROW = 2 * K  # bytes
X, RES, H, Y, W = (i << 32 for i in range(1, 6))


def call(m=M, x=X, ldx=K, res=None, ldr=K, h=None, ldh=K, y=Y, ldy=K, q=None):
    return _abi.lib().tpdq_rmsnorm(x, ldx, res, ldr, W, 1e-5, m, K, 0, h, ldh, None if q else y, ldy,
                                   ctypes.byref(q) if q else None, None)


def mx(codes, scales, ld_c=K, ld_s=16):
    return _abi.Mx(codes, ld_c, scales, ld_s, M, K, _abi.MX_FP8, _abi.MX_ROWS)


SHIFTS = [16, ROW - 16, ROW, 3 * ROW, -16, -3 * ROW]  # rows that meet, all or some of them
RH = dict(res=RES, h=H)


@needs_no_gpu
@pytest.mark.parametrize("d", SHIFTS)
def test_outputs_that_meet_are_refused(d):
    assert call(**RH, y=H + d) == _abi.ERR_SHAPE
    assert call(**RH, q=mx(H + d, Y, ld_c=ROW)) == _abi.ERR_SHAPE
    # scales: 16 bytes a row, 64 in all
    assert call(**RH, q=mx(Y, H + max(d, -48))) == _abi.ERR_SHAPE


@needs_no_gpu
@pytest.mark.parametrize("d", SHIFTS)
def test_an_output_over_a_part_of_an_input_is_refused(d):
    assert call(y=X + d) == _abi.ERR_SHAPE                      # another workgroup's rows
    assert call(**RH, y=RES + d) == _abi.ERR_SHAPE
    assert call(res=RES, h=X + d) == _abi.ERR_SHAPE
    assert call(res=RES, h=RES + d) == _abi.ERR_SHAPE


@needs_no_gpu
def test_the_same_address_with_other_rows_is_refused():
    assert call(y=X, ldy=K + 8) == _abi.ERR_SHAPE and call(y=X, ldx=K + 8) == _abi.ERR_SHAPE
    assert call(**RH, y=RES, ldy=2 * K) == _abi.ERR_SHAPE
    assert call(res=RES, h=RES, ldh=2 * K) == _abi.ERR_SHAPE and call(res=RES, h=X, ldx=2 * K) == _abi.ERR_SHAPE
    assert call(**RH, y=H, ldy=2 * K) == _abi.ERR_SHAPE


# The calls below pass the checks: without a GPU their launch fails, or none is made.
TAKEN = [dict(y=X), dict(res=RES, h=RES), dict(res=RES, h=X), dict(**RH, y=X), dict(res=RES, h=X, y=RES),
         dict(res=RES, h=RES, y=X), dict(res=X, h=X), dict(m=1, y=X, ldy=4 * K), dict(m=1, res=RES, h=RES, ldh=8 * K),
         # columns of one buffer, side by side
         dict(ldx=2 * K, y=X + ROW, ldy=2 * K), dict(ldx=3 * K, res=X + ROW, ldr=3 * K, h=X + ROW, ldh=3 * K, y=X + 2 * ROW, ldy=3 * K),
         # one behind the other
         dict(y=X + M * ROW), dict(**RH, y=H + M * ROW), dict(**RH, y=H - M * ROW), dict(m=1, y=X + ROW),
         dict(**RH, q=mx(H + M * ROW, H - 64))]


@needs_no_gpu
@pytest.mark.parametrize("kw", TAKEN)
def test_other_shared_memory_is_taken(kw):
    assert call(**kw) == _abi.ERR_HIP


@pytest.mark.gpu
def test_shared_memory_gives_the_same_bits():
    import torch
    import paper_2402_04925_amd as tpdq
    from tests import gpu_util as u
    dev = u.torch_dev()
    rows, cols = 300, 520
    g = torch.Generator().manual_seed(1)
    src = torch.randn(rows, 3 * cols, generator=g).to(torch.bfloat16).to(dev)
    w = torch.randn(cols, generator=g).to(torch.bfloat16).to(dev)
    x, res = src[:, :cols], src[:, cols:2 * cols]
    want_y, want_h = tpdq.rmsnorm(x, w, 1e-5, residual=res)

    def parts():
        buf = src.clone()
        return [buf[:, i * cols:(i + 1) * cols] for i in range(3)]
    for pick in (lambda p: (p[2], p[1]), lambda p: (p[0], p[1]), lambda p: (p[1], p[0]), lambda p: (p[2], p[0])):
        p = parts()
        out, h = pick(p)
        y, h = tpdq.rmsnorm(p[0], w, 1e-5, residual=p[1], residual_out=h, out=out)
        assert torch.equal(y, want_y) and torch.equal(h, want_h)
    p = parts()
    with pytest.raises(tpdq.TpdqError):
        tpdq.rmsnorm(p[0], w, 1e-5, residual=p[1], residual_out=p[2], out=p[2])
    with pytest.raises(tpdq.TpdqError):
        tpdq.rmsnorm(src[:-1, :cols], w, 1e-5, out=src[1:, :cols])
    assert torch.equal(tpdq.rmsnorm(x, w, 1e-5, residual=res)[0], want_y)
