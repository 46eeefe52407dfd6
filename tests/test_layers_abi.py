"""Refusals of the layers' and histories' entry points that need no GPU: they come before anything is allocated or launched."""
import ctypes as C

import pytest

from paper_2210_15458_amd import binding


@pytest.fixture(scope="module")
def lib():
    return binding.lib()


def refused(lib, rc, *words, code=1):
    text = lib.as_last_error(None)
    assert rc == code and all(w in text for w in words), (rc, text)


def test_null_context(lib):
    refused(lib, lib.as_linear(None, None, None, 1, 1, None, 0, None, None, 1, 0), b"ctx")
    refused(lib, lib.as_shape_logits(None, None, 1, 1, None, None, 1), b"ctx")
    refused(lib, lib.as_history_set(None, None, 1, None, 1, 1, None, None, None, 0, 1, None, 0, 0, None), b"ctx")
    refused(lib, lib.as_history_add(None, None, 1, None, 1, 1, None, None), b"ctx")


def test_layer_arguments(lib):
    out, W = C.c_void_p(), 4096              # (an address that is looked at but never followed)
    make = lambda *a: lib.as_layer_create(C.byref(out), *a)  # noqa: E731
    refused(lib, lib.as_layer_create(None, W, 8, None, 4, 8, 1.0, 0, 0.0, 1), b"out")
    refused(lib, make(None, 8, None, 4, 8, 1.0, 0, 0.0, 1), b"W is NULL")
    refused(lib, make(W, 8, None, 0, 8, 1.0, 0, 0.0, 1), b"n or k")
    refused(lib, make(W, 8, None, 4, (1 << 21) + 1, 1.0, 0, 0.0, 1), b"n or k")
    refused(lib, make(W, 7, None, 4, 8, 1.0, 0, 0.0, 1), b"ldw")
    refused(lib, make(W, 8, None, 4, 8, 1.0, 0, 0.0, 5), b"dtype")
    refused(lib, make(W, 8, None, 4, 8, 1.0, 6, 0.0, 1), b"activation")
    refused(lib, make(W, 8, None, 4, 8, 1.0, -1, 0.0, 1), b"activation")
    refused(lib, make(W, 8, None, 4, 8, float("nan"), 0, 0.0, 1), b"scale")
    for cap in (0.0, -1.0, float("inf"), float("nan"), 1e-44):
        refused(lib, make(W, 8, None, 4, 8, 1.0, 5, cap, 1), b"cap")
    refused(lib, make(W + 1, 8, None, 4, 8, 1.0, 0, 0.0, 1), b"aligned")
    refused(lib, make(W, 8, W + 2, 4, 8, 1.0, 0, 0.0, 0), b"aligned")
    assert not out.value
    assert lib.as_layer_destroy(None) == 0


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    import torch
    with pytest.raises(TypeError):
        binding.Layer(torch.zeros(4, 8))
    with pytest.raises(ValueError, match="activation"):
        binding.Layer(torch.zeros(4, 8), act="tanh")
    with pytest.raises(TypeError):
        binding.Shaping(2, 64, seen=torch.zeros(2, 2, dtype=torch.int32))
