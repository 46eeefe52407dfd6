"""Members of a shaping or a history that stand for nothing are not read: ids of a table that is not there, lengths of no tokens.
(Their addresses lie on no element here; the calls are those of full members otherwise.)"""
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import problem

pytestmark = pytest.mark.gpu


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


def idle_ids(rows, V):
    """A shaping of nothing, with ids."""
    s = B.Shaping(rows, V, bias_ids=ints(2 * rows), mask_ids=ints(2 * rows))
    s._c.bias_ids += 1
    s._c.mask_ids += 2
    return s


# (7, 8, 9 are for up to 16 rows)
@pytest.mark.parametrize("form,rows", [(f, 9) for f in range(1, 10)] + [(f, 300) for f in range(1, 7)])
def test_ids_of_no_table_in_a_layer(form, rows):
    k, n = 128, 500
    x, W, b, _ = problem(rows, k, n, torch.bfloat16, torch.bfloat16, seed=form)
    ctx, layer = B.Ctx(rows, 16, torch.float32), B.Layer(W, bias=b)
    ctx.set_tuning("linear_shape", form)
    out, plain = (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.as_linear(ctx, layer, x, out, shaping=idle_ids(rows, n))
    B.as_linear(ctx, layer, x, plain)
    assert torch.equal(out, plain)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ids_of_no_table_on_logits(dtype):
    rows, V = 4, 100
    x = torch.randn(rows, V, device="cuda").to(dtype)
    out = torch.empty_like(x)
    B.as_shape_logits(B.Ctx(rows, V, dtype), x, idle_ids(rows, V), out)
    assert torch.equal(out, x)


def test_lengths_of_no_tokens():
    rows, V = 4, 100
    ctx, seen, lens = B.Ctx(rows, V, torch.float32), ints(rows, 4), ints(16)
    assert B.lib().as_history_set(ctx._h, seen.data_ptr(), 4, None, 0, rows, None, None, None, 0, 1, None, 0, 0, lens.data_ptr() + 1) == 0
    assert not bool(seen.any())
