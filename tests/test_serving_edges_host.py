"""Host checks of the binding where a part of torch that it uses is not there."""
import importlib.util

import pytest
import torch

from paper_2112_02194_amd import binding as als


class PlainStream:
    cuda_stream = 77


@pytest.mark.parametrize("missing", ["_cuda_getDevice", "_cuda_getCurrentRawStream"])
def test_the_stream_handle_without_the_short_way(monkeypatch, missing):
    """Without torch's internal functions the handle comes from the public torch.cuda.current_stream()."""
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: PlainStream())
    monkeypatch.delattr(torch._C, missing, raising=False)
    spec = importlib.util.spec_from_file_location("binding_of_another_torch", als.__file__)
    module = importlib.util.module_from_spec(spec)
    monkeypatch.setitem(__import__("sys").modules, spec.name, module)
    spec.loader.exec_module(module)
    assert module._stream() == 77


def test_the_stream_handle_by_the_short_way(monkeypatch):
    monkeypatch.setattr(als, "_current_device", lambda: 3)
    monkeypatch.setattr(als, "_raw_stream", lambda device: 100 + device)
    assert als._stream() == 103
