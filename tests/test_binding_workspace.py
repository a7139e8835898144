"""Workspaces that the kernels must not be given: the binding refuses them before the library is called (no GPU needed)."""
import pytest
import torch


class OnDevice:
    """What the binding looks at in a tensor, of one that claims to be the device's."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, *shape, dtype=torch.float16, gap=False):
        self.t = torch.empty(tuple(n * (1 + gap) for n in shape), dtype=dtype)[tuple(slice(None, None, 1 + gap) for _ in shape)]
        self.shape, self.dtype, self.nbytes = self.t.shape, dtype, self.t.nbytes

    def __getattr__(self, name):
        return getattr(self.t, name)


class Library:
    """Stands for the library: nothing may be called."""
    def __getattr__(self, name):
        raise AssertionError(name + " was called")


@pytest.fixture()
def gs(monkeypatch):
    from paper_2502_11407_amd import binding
    monkeypatch.setattr(binding, "lib", Library())
    return binding


@pytest.mark.parametrize("workspace", [torch.empty(4096, dtype=torch.uint8), OnDevice(4096, dtype=torch.uint8, gap=True)], ids=["host", "gaps"])
def test_workspaces_that_are_not_the_device_s(gs, workspace):
    A, B, C = OnDevice(4, 16), OnDevice(16, 8), OnDevice(4, 8, dtype=torch.float32)
    p, f = gs.gemm_problem("f16", 4, 8, 16), torch.float32
    X, W, t, v = OnDevice(4, 16), OnDevice(8, 16), OnDevice(4, dtype=torch.int64), OnDevice(4, dtype=f)
    stream = type("Stream", (), {"cuda_stream": 0})()
    calls = [lambda: gs.gemm(p, A, B, C, workspace=workspace, stream=stream),
             lambda: gs.bmm(p, OnDevice(1, 4, 16), OnDevice(1, 16, 8), OnDevice(1, 4, 8, dtype=f), workspace=workspace, stream=stream),
             lambda: gs.conv2d(gs.conv_problem("f16", 1, 8, 4, 4, 8, 1, 1, 1, 0), A, B, C, workspace=workspace, stream=stream),
             lambda: gs.gemm_fused(p, A, B, C, workspace=workspace, stream=stream),
             lambda: gs.gemm_act_grad(p, A, B, C, OnDevice(4, 8, dtype=f), "relu", workspace=workspace, stream=stream),
             lambda: gs.bias_grad(A, OnDevice(16), workspace=workspace, stream=stream),
             lambda: gs.xent_forward(X, W, t, v, v, workspace=workspace, stream=stream),
             lambda: gs.xent_backward(X, W, t, v, v, X, W, workspace=workspace, stream=stream)]
    for call in calls:
        with pytest.raises(ValueError, match="workspace"):
            call()
