"""Attention: what one row or token asks for changes no bit of what the others get."""
import pytest
import torch

from attend_util import Batch, check
from test_gpu_attend import FORMS, run as attend
from test_gpu_attend_prompts import run as prompts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (72, 4)])
def test_a_steep_row_among_those_of_its_prompt(form, dim, page):
    """Scores sixty times as steep raise what the row's weights are taken relative to in most tiles; its neighbours' stays theirs."""
    b = Batch([(3 * r) % 20 for r in range(80)], dim, 2, page, form, prompts=[400, 130], per=40, seed=11)
    q, one = attend(b, 8)
    other = q.clone()
    other[1] *= 60
    other[41] *= -60
    _, two = attend(b, 8, q=other)
    rest = [r for r in range(80) if r not in (1, 41)]
    assert torch.equal(one[rest], two[rest])
    check(two, other, b, rows=[0, 1, 2, 40, 41, 79])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (72, 4)])
def test_a_steep_token_of_a_prompt(form, dim, page):
    b = Batch([500], dim, 1, page, form, seed=12)
    q, one, offsets = prompts(b, [300], 4)
    other = q.clone()
    other[[7, 150, 299]] *= 60
    _, two, _ = prompts(b, [300], 4, q=other)
    rest = [i for i in range(300) if i not in (7, 150, 299)]
    assert torch.equal(one[rest], two[rest])
    check(two, other, b, offsets=offsets)


@pytest.mark.parametrize("form", FORMS)
def test_other_sequences_lengths(form):
    """Without a window a row's bits go by its own tokens, whatever the other rows of its prompt have."""
    own = [(7 * r) % 30 for r in range(40)]
    b = Batch(own, 64, 2, 16, form, prompts=[300], per=40, seed=13)
    q, one = attend(b, 8)
    b.lens[1:] = torch.tensor([(11 * r) % 3 for r in range(39)], dtype=torch.int32, device="cuda").minimum(b.lens[1:])
    _, two = attend(b, 8, q=q)
    assert torch.equal(one[0], two[0])
