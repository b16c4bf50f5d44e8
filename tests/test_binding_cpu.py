"""What the binding refuses on the host, before the library is called (no GPU)."""
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
