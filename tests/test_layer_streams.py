"""A Layer, as a Model, is made of tensors that the current stream may still be filling: the binding waits for that stream before the library,
which reads them on another, is called (seen here without a GPU, by the order of the calls)."""
import pytest
import torch

from paper_2210_15458_amd import binding as B


class OnGpu(torch.Tensor):
    """A host tensor that says it is on the GPU; its address is handed on, and followed by nobody."""
    is_cuda = property(lambda self: True)


def on_gpu(*shape):
    return torch.zeros(*shape).as_subclass(OnGpu)


class Library:
    def __init__(self, calls):
        self.calls = calls

    def as_layer_create(self, *a):
        self.calls.append("create")
        return 0

    def as_layer_destroy(self, h):
        return 0

    as_model_create_bigram, as_model_destroy = as_layer_create, as_layer_destroy


class Stream:
    def __init__(self, calls):
        self.calls = calls

    def synchronize(self):
        self.calls.append("wait")


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(B, "lib", lambda: Library(seen))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream(seen))
    return seen


@pytest.mark.parametrize("bias", [False, True])
def test_the_current_stream_is_waited_for(calls, bias):
    B.Layer(on_gpu(4, 64), bias=on_gpu(4) if bias else None)
    assert calls == ["wait", "create"]


def test_nothing_is_waited_for_in_vain(calls):
    with pytest.raises(ValueError):
        B.Layer(on_gpu(4, 64), bias=on_gpu(3))
    assert calls == []


def test_a_model_s_too(calls):
    B.Model(on_gpu(8, 64), on_gpu(64, 8))
    assert calls == ["wait", "create"]
