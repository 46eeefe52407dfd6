"""Layers of tensors that a side stream has only just been asked to make."""
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import check, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,k", [(torch.bfloat16, 256), (torch.bfloat16, 250), (torch.float32, 96)])
def test_made_inside_a_side_stream(dtype, k):
    rows, n = 70, 300
    x, W, b, _ = problem(rows, k, n, dtype, dtype, seed=k)
    busy = torch.randn(4096, 4096, device="cuda")
    late_W, late_b = torch.zeros_like(W), torch.zeros_like(b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(8):                   # milliseconds before the weights are there
            busy = (busy @ busy).clamp_(-1.0, 1.0)
        late_W.copy_(W)
        late_b.copy_(b)
        layer, out = B.Layer(late_W, bias=late_b), torch.empty(rows, n, dtype=dtype, device="cuda")
        B.as_linear(B.Ctx(rows, 16, torch.float32), layer, x, out)
    side.synchronize()
    check(out, x, W, b, "none", 1.0, None, (dtype, k))
