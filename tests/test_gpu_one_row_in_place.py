"""One row has no stride: shaped in place, or with the residual in its outputs, it may be given as parts of its memory of different
widths; of several rows the strides have to agree."""
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import check, problem

pytestmark = pytest.mark.gpu


def test_shaped_in_place():
    V = 100
    wide = torch.randn(1, V + 30, device="cuda")
    want = wide.clone()
    want[:, :V] += 2.0
    shaping = B.Shaping(1, V, bias=torch.full((1, V), 2.0, device="cuda"))
    B.as_shape_logits(B.Ctx(1, V, torch.float32), wide, shaping, wide[:, :V])
    assert torch.equal(wide, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_residual_in_place(dtype):
    k, n = 64, 100
    x, W, b, r = problem(1, k, n, dtype, dtype, seed=1, residual=True)
    wide = torch.full((1, n + 30), 7.0, dtype=dtype, device="cuda")
    wide[:, :n] = r
    B.as_linear(B.Ctx(1, 16, torch.float32), B.Layer(W, bias=b), x, wide[:, :n], residual=wide)
    check(wide[:, :n], x, W, b, "none", 1.0, r, dtype)
    assert bool((wide[:, n:] == 7.0).all())


def test_several_rows_are_refused():
    """(the same memory with other strides: one row's outputs would lie in the next one's inputs)"""
    V = 100
    flat = torch.zeros(3 * 130, device="cuda")
    a, b = flat[:260].view(2, 130), flat[:200].view(2, 100)
    with pytest.raises(B.ArithSamplingError, match="in place"):
        B.as_shape_logits(B.Ctx(2, V, torch.float32), a, B.Shaping(2, V), b)
    layer, x = B.Layer(torch.zeros(V, 8, device="cuda")), torch.zeros(2, 8, device="cuda")
    with pytest.raises(B.ArithSamplingError, match="in place"):
        B.as_linear(B.Ctx(2, 16, torch.float32), layer, x, b, residual=a)
