"""Attention: windows as wide as an int holds, and chunks whose first queries lie before their sequence."""
import pytest
import torch

from attend_util import Batch, check
from test_gpu_attend import FORMS, run as attend
from test_gpu_attend_prompts import run as prompts

pytestmark = pytest.mark.gpu

WIDEST = 2 ** 31 - 1


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window,sinks", [(WIDEST, 0), (WIDEST, WIDEST), (WIDEST - 3, 2), (3, 1)])
@pytest.mark.parametrize("new", [9, 200])
def test_more_queries_than_tokens(form, window, sinks, new):
    b = Batch([5, 8], 64, 1, 16, form, seed=3)
    q, out, offsets = prompts(b, [new, 8], 2, window=window, sinks=sinks)
    assert bool((out[:new - 5] == 0).all())
    check(out, q, b, rows=[1], offsets=offsets, window=window, sinks=sinks)
    check(out[new - 5:new], q[new - 5:new], b, rows=[0], offsets=[0, 5], window=window, sinks=sinks)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window,sinks", [(WIDEST, 0), (WIDEST, WIDEST), (WIDEST - 3, 2)])
def test_rows_with_and_without_tokens(form, window, sinks):
    """Among them waves of 32 queries without one, and rows that see nothing."""
    own = [(3 * r) % 7 for r in range(70)]
    b = Batch(own, 64, 1, 16, form, prompts=[0, 90], per=35, seed=4)
    finished = torch.zeros(70, dtype=torch.uint8, device="cuda")
    finished[40:60] = 1
    q, out = attend(b, 4, window=window, sinks=sinks, finished=finished)
    assert bool((out[40:60] == 7).all()) and bool((out[0] == 0).all())
    check(out, q, b, rows=[0, 1, 34, 35, 39, 60, 69], window=window, sinks=sinks)
