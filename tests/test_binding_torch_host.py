"""The binding asks torch for the current device and stream by its private shortcuts where they exist, and works without them."""
import importlib.util
import types

import torch

from paper_2609_39068_b200 import binding


def test_a_torch_without_the_shortcuts(monkeypatch):
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: types.SimpleNamespace(cuda_stream=1000 + dev))
    spec = importlib.util.spec_from_file_location(binding.__name__ + "_again", binding.__file__)
    spec.loader.exec_module(again := importlib.util.module_from_spec(spec))
    assert again._current_device() == 3 and again._stream_handle(2) == 1002
    # a call: on the workspace's device, with that device's stream
    seen = []
    monkeypatch.setattr(again, "_lib", types.SimpleNamespace(se_any=lambda *args: seen.append(args) or 0))
    monkeypatch.setattr(again, "_ptr", lambda t, dtype, name: 4096)
    again._call("se_any", types.SimpleNamespace(get_device=lambda: 3), (), 7)
    assert seen == [(7, 4096, 1003)]
