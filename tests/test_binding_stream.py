"""The handle of the current stream: by torch's own functions for it, which are private, or without them (CPU, fakes)."""
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def binding(monkeypatch):
    from paper_2311_05827_b200 import binding as b
    monkeypatch.setattr(b, "_raw_stream", None)  # and back to what it was
    monkeypatch.setattr(torch.cuda, "init", lambda: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    return b


def test_a_stream_that_is_given(binding):
    assert binding._stream_handle(types.SimpleNamespace(cuda_stream=5)) == 5


def test_current_stream_by_the_private_functions(binding, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    assert binding._stream_handle() == 1003


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_current_stream_where_torch_lacks_one_of_them(binding, monkeypatch, missing):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.delattr(torch._C, missing)
    assert binding._stream_handle() == 77
    assert binding._stream_handle() == 77
