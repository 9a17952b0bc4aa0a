"""The stream that a call takes when it is given none: torch's current one, with and without torch's quick way to it."""
import types

import pytest

import paper_2607_19456_b200 as moa

torch = pytest.importorskip("torch")


@pytest.fixture
def fresh(monkeypatch):
    monkeypatch.setattr(moa, "_current_stream", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=77))
    return monkeypatch


def test_through_the_raw_call(fresh):
    fresh.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 40 + device, raising=False)
    assert moa._stream(None) == 43 and moa._stream(None) == 43


def test_without_the_raw_call(fresh):
    fresh.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert moa._stream(None) == 77


def test_a_stream_that_is_given():
    assert moa._stream(5) == 5 and moa._stream(types.SimpleNamespace(cuda_stream=9)) == 9


@pytest.mark.gpu
def test_the_current_stream():
    assert moa._stream(None) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert moa._stream(None) == side.cuda_stream
