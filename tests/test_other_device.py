"""Tensors of another device than the current one: its default stream's handle would stand for the current device's, and the
kernels would run there."""
import types

import pytest


@pytest.fixture(scope="module")
def m():
    from paper_2606_07618_amd import nvfp4
    return nvfp4


def on(index):
    return types.SimpleNamespace(get_device=lambda: index, device=f"cuda:{index}")


def test_the_default_stream_of_another_device_is_refused(m, monkeypatch):
    monkeypatch.setattr(m, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(m, "_current_device", lambda: 0)
    assert m._stream(on(0)) == 0
    with pytest.raises(ValueError, match="cuda:1"):
        m._stream(on(1))
    monkeypatch.setattr(m, "_current_device", lambda: 1)
    assert m._stream(on(1)) == 0
    with pytest.raises(ValueError, match="cuda:0"):
        m._stream(on(0))


def test_a_stream_of_its_own_names_its_device(m, monkeypatch):
    monkeypatch.setattr(m, "_raw_stream", lambda index: 0x7000 + index)
    monkeypatch.setattr(m, "_current_device", lambda: 0)
    assert m._stream(on(1)) == 0x7001 and m._stream(on(0)) == 0x7000
    with pytest.raises(ValueError, match="cuda device"):
        m._stream(on(-1))


@pytest.mark.gpu
def test_the_current_device(m):
    import torch
    x = torch.zeros((2, 16), device="cuda:0")
    assert m._stream(x) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert m._stream(x) == side.cuda_stream
