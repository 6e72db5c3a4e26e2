"""Where the binding gets the device and the stream of a call from: torch's public names, or a quicker one where torch has it."""
import importlib.util
from types import SimpleNamespace

import pytest
import torch

from paper_2603_08026_amd import binding


def test_without_the_quick_name(monkeypatch):
    """A torch that lacks it is asked the public way.  No GPU needed."""
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: SimpleNamespace(cuda_stream=100 + d))
    spec = importlib.util.spec_from_file_location("paper_2603_08026_amd.binding_again", binding.__file__)
    again = importlib.util.module_from_spec(spec)
    monkeypatch.setitem(__import__("sys").modules, spec.name, again)  # (dataclasses look their module up)
    spec.loader.exec_module(again)
    assert again._device() == 3 and again._raw_stream(3) == 103


@pytest.mark.gpu
def test_the_stream_is_the_current_one():
    dev = binding._device()
    assert dev == torch.cuda.current_device()
    assert binding._raw_stream(dev) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert binding._raw_stream(dev) == side.cuda_stream
    assert binding._raw_stream(dev) == torch.cuda.current_stream().cuda_stream != side.cuda_stream
