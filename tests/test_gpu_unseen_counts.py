"""Counts of tokens whose seen bit is not set say nothing, whatever stands there, whether few of a row's columns are seen (their
counts alone are looked up) or most (all are read)."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_shaping import inputs, pack

pytestmark = pytest.mark.gpu

NAMES = ("repetition", "presence", "frequency")


def pair(rows, V, share):
    """The same shaping with zeros and with anything in the counts of what is not seen."""
    rng = np.random.default_rng(V)
    p = inputs(rows, V, seed=V)
    p["seen"] = rng.random((rows, V)) < share
    clean = np.where(p["seen"], rng.integers(0, 5, (rows, V)), 0).astype(np.int32)
    dirty = np.where(p["seen"], clean, rng.integers(-2 ** 31, 2 ** 31, (rows, V))).astype(np.int32)
    fixed = {n: torch.from_numpy(p[n]).cuda() for n in NAMES}
    return [B.Shaping(rows, V, seen=pack(p["seen"]), counts=torch.from_numpy(c).cuda(), **fixed) for c in (clean, dirty)]


@pytest.mark.parametrize("rows,V", [(5, 2050), (70, 33333)])
@pytest.mark.parametrize("share", [0.01, 0.9])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits(rows, V, share, dtype):
    x = torch.randn(rows, V, device="cuda").to(dtype)
    a, b = torch.empty_like(x), torch.empty_like(x)
    ctx = B.Ctx(rows, V, dtype)
    for s, out in zip(pair(rows, V, share), (a, b)):
        B.as_shape_logits(ctx, x, s, out)
    assert torch.equal(a, b)


@pytest.mark.parametrize("form,rows", [(f, 300) for f in range(1, 7)] + [(f, 16) for f in (7, 8, 9)])
@pytest.mark.parametrize("share", [0.01, 0.9])
def test_layers(form, rows, share):
    k, n = 128, 1001
    W, x = torch.randn(n, k, device="cuda").to(torch.bfloat16), torch.randn(rows, k, device="cuda").to(torch.bfloat16)
    ctx, layer = B.Ctx(rows, 16, torch.float32), B.Layer(W)
    ctx.set_tuning("linear_shape", form)
    a, b = (torch.empty(rows, n, device="cuda") for _ in range(2))
    for s, out in zip(pair(rows, n, share), (a, b)):
        B.as_linear(ctx, layer, x, out, shaping=s)
    assert torch.equal(a, b)
