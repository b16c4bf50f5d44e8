"""The binding's own work on the GPU: workspaces and refusals of public calls."""
import pytest

import paper_2402_04925_amd as tpdq
from paper_2402_04925_amd import inputs
from tests import gpu_util as u

pytestmark = pytest.mark.gpu


def test_workspace_without_a_device_and_of_the_host():
    import torch
    dev = u.torch_dev()
    f16 = torch.float16
    x = torch.randn(20, 512, generator=torch.Generator().manual_seed(1)).to(f16).to(dev)
    mx = [tpdq.mx_pack(tpdq.mx_quantize(torch.randn(512, 512, generator=torch.Generator().manual_seed(i)).to(f16).to(dev),
                                        tpdq.MX_FP4)) for i in (2, 3)]
    q = tpdq.mx_quantize(x, tpdq.MX_FP8)
    w, _ = inputs.make_custom(512, 256, 0, 128, seed=4)
    w = u.layer_to_dev(w, dev)
    calls = [lambda ws: tpdq.mx_mlp_shard(q, mx[0], mx[1], f16, workspace=ws),
             lambda ws: tpdq.w4a16_gemm(x, w, tpdq.PATH_ACTORDER, workspace=ws)]
    for call in calls:
        ws = tpdq.Workspace()
        assert torch.equal(call(ws), call(None)) and ws.buf.device == dev
        with pytest.raises(ValueError, match="workspace"):
            call(tpdq.Workspace("cpu"))
