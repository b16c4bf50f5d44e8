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


def test_graph_outlives_the_growth_of_its_workspace():
    import torch
    dev = u.torch_dev()
    f16 = torch.float16
    rand = lambda i, *s: torch.randn(*s, generator=torch.Generator().manual_seed(i)).to(f16).to(dev)
    up, down = (tpdq.mx_pack(tpdq.mx_quantize(rand(i, 512, 512), tpdq.MX_FP4)) for i in (1, 2))
    w, _ = inputs.make_custom(512, 512, 512, 128, seed=4)
    w = u.layer_to_dev(w, dev)
    x = rand(3, 40, 512)
    for call in (lambda ws: tpdq.mx_mlp_shard(tpdq.mx_quantize(x, tpdq.MX_FP8), up, down, f16, workspace=ws),
                 lambda ws: tpdq.w4a16_gemm(x, w, tpdq.PATH_ACTORDER, workspace=ws)):
        ws = tpdq.Workspace(dev)
        want = call(ws).clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = call(ws)
        ws.get(64 << 20)
        # memory of the first buffer's size, as the allocator would hand it out again
        others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device=dev) for _ in range(8)]
        for _ in range(3):
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and all(bool((o == 7).all()) for o in others)
            out.zero_()
