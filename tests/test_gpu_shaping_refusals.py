"""Arrays of a shaping or a history that do not lie on whole elements, and numbers of rows that mean nothing, are refused before
anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS, V = 4, 100


def refused(ctx, rc, words):
    text = (B.lib().as_last_error(ctx._h) or b"").decode()
    assert rc == 1 and words in text, (rc, text)


def ints(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


@pytest.mark.parametrize("name", ["repetition", "presence", "frequency", "bias_ids", "mask_ids"])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_a_shaping_s_rows(name, shift):
    ctx = B.Ctx(ROWS, V, torch.float32)
    ones = torch.ones(2 * ROWS, device="cuda")
    s = B.Shaping(ROWS, V, seen=ints(ROWS, 4), counts=ints(ROWS, V), repetition=ones, presence=ones, frequency=ones,
                  bias=torch.zeros(3, V, device="cuda"), bias_ids=ints(2 * ROWS), mask=ints(3, 4), mask_ids=ints(2 * ROWS))
    x = torch.randn(ROWS, V, device="cuda")
    out = torch.full((ROWS, V), 7.0, device="cuda")
    setattr(s._c, name, getattr(s._c, name) + shift)
    refused(ctx, B.lib().as_shape_logits(ctx._h, x.data_ptr(), ROWS, V, C.byref(s._c), out.data_ptr(), V), "aligned")
    layer, y = B.Layer(torch.randn(V, 8, device="cuda")), torch.randn(ROWS, 8, device="cuda")
    refused(ctx, B.lib().as_linear(ctx._h, layer._h, y.data_ptr(), ROWS, 8, None, 0, C.byref(s._c), out.data_ptr(), V, B.AS_F32), "aligned")
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("name,shift", [("prompts", 2), ("offsets", 4), ("tokens", 1), ("lens", 3)])
def test_a_history_s_lists(name, shift):
    ctx = B.Ctx(ROWS, V, torch.float32)
    seen, counts = ints(ROWS, 4), ints(ROWS, V)
    t = {"prompts": ints(64), "offsets": torch.arange(16, device="cuda"), "tokens": ints(ROWS, 9), "lens": ints(16)}
    at = {k: v.data_ptr() + (shift if k == name else 0) for k, v in t.items()}
    refused(ctx, B.lib().as_history_set(ctx._h, seen.data_ptr(), 4, counts.data_ptr(), V, ROWS, None, at["prompts"], at["offsets"], 60, 1,
                                        at["tokens"], 9, 8, at["lens"]), "aligned")
    if name == "tokens":
        refused(ctx, B.lib().as_history_add(ctx._h, seen.data_ptr(), 4, counts.data_ptr(), V, ROWS, at["tokens"], None), "aligned")
    torch.cuda.synchronize()
    assert not bool(seen.any()) and not bool(counts.any())


@pytest.mark.parametrize("per", [0, -1, -7])
def test_rows_per_prompt(per):
    ctx = B.Ctx(ROWS, V, torch.float32)
    seen = ints(ROWS, 4)
    with pytest.raises(B.ArithSamplingError, match="rows_per_prompt"):
        B.as_history_set(ctx, seen, None, ints(5), torch.zeros(9, dtype=torch.int64, device="cuda"), per)
    assert not bool(seen.any())
