"""Refusals of the cache's and the attention's entry points and of their binding that need no GPU."""
import ctypes as C

import pytest
import torch

from paper_2210_15458_amd import binding as B


class OnGpu(torch.Tensor):
    """A host tensor that says it is on the GPU; its address is handed on, and followed by nobody."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def test_null_context():
    lib = B.lib()
    c, s = B._Cache(), B._Sequences()
    for rc in (lib.as_cache_add(None, C.byref(c), C.byref(s), 1, None, 1, None, 1, 1, None),
               lib.as_attend(None, C.byref(c), C.byref(s), 1, None, 1, 1, 1.0, 0, 0, None, 1),
               lib.as_attend_prompts(None, C.byref(c), C.byref(s), 1, None, 1, 1, None, 1, 1.0, 0, 0, None, 1)):
        assert rc == 1 and b"ctx" in lib.as_last_error(None)


def test_caches():
    B.Cache(on_gpu(4, 2, 16, 64), on_gpu(4, 2, 16, 64))
    both = on_gpu(4, 2, 2, 16, 64)
    c = B.Cache(both[:, 0], both[:, 1])
    assert c._c.page_ld == 2 * 2 * 16 * 64 and c._c.pages == 4 and c._c.page_size == 16
    with pytest.raises(TypeError, match="GPU"):
        B.Cache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64))
    with pytest.raises(ValueError, match="pages"):
        B.Cache(on_gpu(4, 16, 64), on_gpu(4, 16, 64))
    with pytest.raises(ValueError, match="one shape"):
        B.Cache(on_gpu(4, 2, 16, 64), on_gpu(4, 2, 16, 72))
    with pytest.raises(ValueError, match="one shape"):
        B.Cache(on_gpu(4, 2, 16, 64), on_gpu(4, 2, 16, 64, dtype=torch.float32))
    with pytest.raises(ValueError, match="one shape"):
        B.Cache(on_gpu(4, 2, 16, 64), both[:, 0])
    with pytest.raises(ValueError, match="contiguous"):
        B.Cache(on_gpu(4, 16, 2, 64).transpose(1, 2), on_gpu(4, 16, 2, 64).transpose(1, 2))
    with pytest.raises(TypeError, match="storage dtype"):
        B.Cache(on_gpu(4, 2, 16, 64, dtype=torch.float16), on_gpu(4, 2, 16, 64, dtype=torch.float16))


def test_sequences():
    i32 = dict(dtype=torch.int32)
    s = B.Sequences(3, on_gpu(3, 5, **i32), on_gpu(3, **i32), on_gpu(2, 7, **i32), on_gpu(2, **i32), 2)
    assert s._c.table_ld == 5 and s._c.prompt_table_ld == 7 and s._c.rows_per_prompt == 2
    with pytest.raises(ValueError, match="lengths"):
        B.Sequences(3, on_gpu(3, 5, **i32))
    with pytest.raises(ValueError, match="lengths"):
        B.Sequences(3, on_gpu(3, 5, **i32), on_gpu(3, **i32), prompt_lens=on_gpu(2, **i32))
    with pytest.raises(ValueError, match="lens"):
        B.Sequences(3, on_gpu(3, 5, **i32), on_gpu(2, **i32))
    with pytest.raises(TypeError, match="int32"):
        B.Sequences(3, on_gpu(3, 5, dtype=torch.int64), on_gpu(3, **i32))
    with pytest.raises(ValueError, match="table"):
        B.Sequences(3, on_gpu(2, 5, **i32), on_gpu(3, **i32))
    with pytest.raises(ValueError, match="contiguous"):
        B.Sequences(3, on_gpu(3, 6, **i32)[:, :5], on_gpu(3, **i32))
    with pytest.raises(ValueError, match="prompt"):
        B.Sequences(5, on_gpu(5, 5, **i32), on_gpu(5, **i32), on_gpu(2, 7, **i32), on_gpu(2, **i32), 2)
    with pytest.raises(ValueError, match="rows_per_prompt"):
        B.Sequences(5, prompt_table=on_gpu(2, 7, **i32), prompt_lens=on_gpu(2, **i32), rows_per_prompt=0)
    with pytest.raises(TypeError, match="uint8"):
        B.Sequences(3, on_gpu(3, 5, **i32), on_gpu(3, **i32), finished=on_gpu(3, **i32))


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


class Stream:
    device_index = 0


class Ctx:
    _h, stream = None, Stream()


@pytest.fixture
def library(monkeypatch):
    made = Library()
    monkeypatch.setattr(B, "lib", lambda: made)
    monkeypatch.setattr(B, "_lib", made)
    return made


def test_rows_of_heads(library):
    """What the calls hand on of q, out, k and v: rows apart, heads as a dimension; and what they refuse."""
    i32 = dict(dtype=torch.int32)
    cache = B.Cache(on_gpu(4, 2, 16, 64), on_gpu(4, 2, 16, 64))
    seqs = B.Sequences(3, on_gpu(3, 5, **i32), on_gpu(3, **i32))
    qkv, out = on_gpu(3, 8 * 64), on_gpu(3, 4 * 64)
    B.as_attend(Ctx, cache, seqs, qkv[:, :256], out)
    B.as_attend(Ctx, cache, seqs, qkv.view(3, 8, 64)[:, :4], out.view(3, 4, 64), window=7, sinks=2)
    (_, one), (_, two) = library.calls
    assert one[4:7] == (qkv.data_ptr(), 512, 4) and one[8:] == (0, 0, out.data_ptr(), 256) and two[4:7] == one[4:7] and two[8:10] == (7, 2)
    assert abs(one[7] - 0.125) < 1e-9
    B.as_cache_add(Ctx, cache, seqs, qkv[:, 256:384], qkv.view(3, 8, 64)[:, 6:])
    name, add = library.calls[-1]
    assert name == "as_cache_add" and add[4:] == (qkv.data_ptr() + 512, 512, qkv.data_ptr() + 768, 512, 3, None)
    calls = len(library.calls)
    with pytest.raises(ValueError, match="q has"):
        B.as_attend(Ctx, cache, seqs, on_gpu(3, 100), out)
    with pytest.raises(ValueError, match="out"):
        B.as_attend(Ctx, cache, seqs, qkv[:, :256], on_gpu(3, 128))
    with pytest.raises(ValueError, match="q is 2"):
        B.as_attend(Ctx, cache, seqs, qkv[:2, :256], out)
    with pytest.raises(TypeError, match="q must be"):
        B.as_attend(Ctx, cache, seqs, on_gpu(3, 256, dtype=torch.float32), out)
    with pytest.raises(ValueError, match="contiguous rows"):
        B.as_attend(Ctx, cache, seqs, on_gpu(256, 3).t(), out)
    with pytest.raises(ValueError, match="heads one behind the other"):
        B.as_attend(Ctx, cache, seqs, on_gpu(4, 3, 64).transpose(0, 1), out)
    with pytest.raises(TypeError, match="GPU"):
        B.as_cache_add(Ctx, cache, seqs, torch.zeros(3, 128, dtype=torch.bfloat16), qkv[:, :128])
    with pytest.raises(TypeError, match="offsets"):
        B.as_attend_prompts(Ctx, cache, seqs, qkv[:, :256], on_gpu(4, **i32), out)
    with pytest.raises(ValueError, match="offsets"):
        B.as_attend_prompts(Ctx, cache, seqs, qkv[:, :256], on_gpu(3, dtype=torch.int64), out)
    assert len(library.calls) == calls


def test_one_device(library):
    class Elsewhere(OnGpu):
        def get_device(self):
            return 1

    i32 = dict(dtype=torch.int32)
    cache = B.Cache(on_gpu(4, 2, 16, 64), on_gpu(4, 2, 16, 64))
    seqs = B.Sequences(3, on_gpu(3, 5, **i32), on_gpu(3, **i32))
    away = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype).as_subclass(Elsewhere)  # noqa: E731
    with pytest.raises(ValueError, match="one device"):
        B.Sequences(3, on_gpu(3, 5, **i32), away(3, **i32))
    with pytest.raises(ValueError, match="one device"):
        B.as_attend(Ctx, cache, B.Sequences(3, away(3, 5, **i32), away(3, **i32)), on_gpu(3, 256), on_gpu(3, 256))
    with pytest.raises(ValueError, match="one device"):
        B.as_attend(Ctx, B.Cache(away(4, 2, 16, 64), away(4, 2, 16, 64)), seqs, on_gpu(3, 256), on_gpu(3, 256))
    with pytest.raises(ValueError, match="q must be on"):
        B.as_attend(Ctx, cache, seqs, away(3, 256), on_gpu(3, 256))
    with pytest.raises(ValueError, match="offsets must be on"):
        B.as_attend_prompts(Ctx, cache, seqs, on_gpu(3, 256), away(4, dtype=torch.int64), on_gpu(3, 256))
    assert not library.calls
