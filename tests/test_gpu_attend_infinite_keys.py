"""A visible key with an infinity whose score is -inf has no weight, whatever the rows' length: what rows are padded with adds nothing."""
import math

import pytest
import torch

from attend_util import Batch, attention, seen_by
from test_gpu_attend import FORMS, run as attend
from test_gpu_attend_prompts import run as prompts

pytestmark = pytest.mark.gpu

DIMS = [(64, 16), (128, 16), (256, 16), (8, 16), (56, 16), (72, 16), (72, 4), (80, 1), (96, 16), (104, 16), (120, 8), (136, 16), (192, 16), (200, 16), (248, 4)]


def check(out, q, b, r, i, at, gone):
    k, v = b.tokens(r)
    see = seen_by(at, k.shape[1], 0, 0)
    for t in gone:
        see[t] = False
    want, far = attention(q[i].view(-1, b.dim), k, v, see, b.dim ** -0.5)
    d = (out[i].view(-1, b.dim).double() - want).abs()
    assert bool((d <= far).all()), (r, i, float((d / far).nan_to_num(nan=math.inf).max()))


def without_weight(b, r, t, component):
    p, i = b.place(r, t)
    b.k[p, :, i, component] = -math.inf


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dim,page", DIMS)
@pytest.mark.parametrize("last", [False, True])
def test_rows(form, dim, page, last):
    """Of a prompt and of rows' own; the infinity in the first piece of a row, or in its last value."""
    b = Batch([30, 0, 5, 70] * 5, dim, 2, page, form, prompts=[130], per=20, seed=dim)
    at = dim - 1 if last else 3
    without_weight(b, 0, 77, at)                  # (of the prompt)
    without_weight(b, 3, 130 + 33, at)            # (row 3's own)
    q = torch.randn(20, 2, 4, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    q[..., at] = q[..., at].abs() + 0.1
    q = q.view(20, -1).to(b.dtype)
    _, out = attend(b, 8, q=q)
    for r in (0, 1, 2, 3, 19):
        check(out, q, b, r, r, 130 + b.own[r] - 1, [77, 163] if r == 3 else [77])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dim,page", DIMS)
def test_prompts(form, dim, page):
    b = Batch([100], dim, 1, page, form, seed=dim)
    for t in (2, 40):
        without_weight(b, 0, t, 3)
    q = torch.randn(90, 4, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    q[..., 3] = q[..., 3].abs() + 0.1
    q = q.view(90, -1).to(b.dtype)
    _, out, _ = prompts(b, [90], 4, q=q, behind=0)
    for i in (0, 1, 29, 30, 31, 60, 89):
        check(out, q, b, 0, i, 10 + i, [2, 40])
