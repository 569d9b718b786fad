"""CPU-only checks of what the operators around the time-step loop demand of their tensors' devices: stand-ins for tensors, and a library that only tells that it was called."""
import types

import pytest
import torch

from paper_2412_07752_amd import api


class Tensor:
    """What the Python part of a call looks at."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, device=0):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", device)

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 4096


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library; device 0 is the current one."""
    made = []
    monkeypatch.setattr(api, "_native", None)
    monkeypatch.setattr(api, "lib", lambda: types.SimpleNamespace(flashrnn_grad_clip_workspace_bytes=lambda n: 16, flashrnn_grad_clip=lambda *a: made.append(a) or api.FLASHRNN_OK))
    monkeypatch.setattr(api, "_stream", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return made


def test_clipping_takes_its_tensors_and_its_workspace_on_the_current_device(calls):
    norm, ws = Tensor(1), Tensor(16, dtype=torch.uint8)
    far_ws, far_norm, g, far_g = Tensor(16, dtype=torch.uint8, device=1), Tensor(1, device=1), Tensor(5), Tensor(5, device=1)
    assert api.flashrnn_grad_clip([g], 1.0, norm=norm, workspace=ws) is norm and api.flashrnn_grad_clip([], 1.0, norm=norm, workspace=ws) is norm and len(calls) == 2
    for grads, n, w in (([g], norm, far_ws), ([], norm, far_ws), ([far_g], norm, ws), ([], far_norm, far_ws), ([far_g], far_norm, far_ws)):
        with pytest.raises(ValueError, match="is on cuda:1|are on cuda:1"):
            api.flashrnn_grad_clip(grads, 1.0, norm=n, workspace=w)
    with pytest.raises(ValueError, match="out is on cuda:1"):
        api.flashrnn_grad_clip([g], 1.0, out=[far_g], norm=norm, workspace=ws)
    assert len(calls) == 2
