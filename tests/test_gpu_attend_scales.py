"""Attention with the largest and smallest scales: those whose product with log2(e) is no number are refused, others weigh as any."""
import pytest
import torch

from attend_util import Batch
from paper_2210_15458_amd import binding as B
from test_gpu_attend import FORMS, run as attend
from test_gpu_attend_far_scores import check, keys, queries, scattered
from test_gpu_attend_prompts import run as prompts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("scale", [2.3e38, -2.3e38, 1e-30, 1e-42, -1e-45])
def test_results(form, scale):
    b = Batch([(5 * r) % 23 for r in range(40)], 128, 1, 16, form, prompts=[500, 70], per=20, seed=1)
    keys(b, scattered(1))
    q = queries(40, 8, 128, b.dtype, 10)
    _, out = attend(b, 8, q=q, scale=scale)
    check(out, q, b, scale, [0, 1, 2, 3, 19, 20, 38, 39])
    b = Batch([170, 40], 64, 1, 16, form, seed=1)
    keys(b, scattered(1))
    q = queries(200, 4, 64, b.dtype, 10)
    _, out, offsets = prompts(b, [160, 40], 4, q=q, scale=scale, behind=0)
    check(out, q, b, scale, [0, 1], offsets=offsets)


@pytest.mark.parametrize("scale", [2.4e38, -3.4e38])
def test_refusals(scale):
    b = Batch([40, 3], 64, 1, 16, "bf16")
    ctx, cache, seqs = B.Ctx(4, 100), B.Cache(b.k, b.v), B.Sequences(2, b.table, b.lens)
    q = torch.randn(2, 64, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    for call in (lambda: B.as_attend(ctx, cache, seqs, q, out, scale=scale),
                 lambda: B.as_attend_prompts(ctx, cache, seqs, q, torch.tensor([0, 1, 2], device="cuda"), out, scale=scale)):
        with pytest.raises(B.ArithSamplingError, match="scale") as e:
            call()
        assert e.value.code == 1
    torch.cuda.synchronize()
    assert bool((out == 7).all())
