"""Attention with scores of any finite size: scores that fp32 holds as they are, so that the formula in 64 bits has the same."""
import pytest
import torch

from attend_util import Batch
from test_gpu_attend import FORMS, run as attend
from test_gpu_attend_prompts import run as prompts

pytestmark = pytest.mark.gpu

FAR = 175 / 128                                   # (eight bits, as bf16 has)
SCALE = 0.3


def keys(b, of):
    """Keys (1, of(first token, tokens), 0, ...) in the slots that hold a token."""
    used = ~b.k.isnan()
    k = torch.zeros_like(b.k)
    k[..., 0] = 1
    for page_list in b.lists:
        for i, p in enumerate(page_list):
            k[p, :, :, 1] = of(i * b.page, b.page).to(b.dtype)
    b.k = torch.where(used, k, b.k)


def queries(n, heads, dim, dtype, power, sign=1.0, steps=None):
    """Queries (sign FAR 2^power, step, 0, ...), every third of a small power: scores of at most 24 bits."""
    q = torch.zeros(n, heads, dim, device="cuda")
    powers = [4 if i % 3 == 0 else power for i in range(n)]      # (by host floats, whose powers of two are exact)
    q[:, :, 0] = torch.tensor([sign * FAR * 2.0 ** p for p in powers], device="cuda")[:, None]
    q[:, :, 1] = torch.tensor([2.0 ** max(p - 22, -1) if steps is None else steps for p in powers], device="cuda")[:, None]
    return q.view(n, -1).to(dtype)


def check(out, q, b, scale, rows, offsets=None):
    """Scores and their differences are exact.  An exponent is a product of the difference and of scale log2(e), which is rounded
    three times: (4.1 |x| + 1) 2^-24 of a weight, and 2^-22 for the exponential's result; a query's sums are scaled anew at most ten times
    (eight scores, or as many tiles as matter; waves and parts), by as much each.  Twice (weights, their sum); sums over n tokens in parts
    (n + 64) 2^-24; bf16 weights 2 u more, as everywhere; the result's rounding u."""
    u = torch.finfo(q.dtype).eps / 2
    for r in rows:
        k, v = b.tokens(r)
        first, last = (r, r + 1) if offsets is None else (offsets[r], offsets[r + 1])
        for i in range(first, last):
            n = k.shape[1] - (last - 1 - i)
            qd = q[i].double().view(b.kv_heads, -1, b.dim)
            s = ((qd[:, :, None, 0] * k[:, None, :n, 0] + qd[:, :, None, 1] * k[:, None, :n, 1]))
            assert torch.equal(s.float().double(), s)
            x = s * float(torch.tensor(scale))
            x = x - x.amax(-1, keepdim=True)
            p = torch.exp(x)
            p = p / p.sum(-1, keepdim=True)
            want = (p.unsqueeze(-1) * v[:, None, :n]).sum(2).reshape(-1, b.dim)
            spread = (p.unsqueeze(-1) * v[:, None, :n].abs()).sum(2).reshape(-1, b.dim)
            each = 10 * ((4.1 * x.abs() + 1) * 2.0 ** -24 + 2.0 ** -22)
            off = ((p * each).unsqueeze(-1) * v[:, None, :n].abs()).sum(2).reshape(-1, b.dim) + (p * each).sum(-1).reshape(-1, 1) * spread
            far = off + ((n + 64) * 2.0 ** -24 + (2 * u if q.dtype == torch.bfloat16 else 0.0)) * spread + u * want.abs() * 1.02 + 1e-30
            d = (out[i].double().view(-1, b.dim) - want).abs()
            assert bool((d <= far).all()), (r, i, float((d / far).nan_to_num(nan=1e9).max()))


def scattered(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda first, n: -torch.randint(0, 8, (n,), device="cuda", generator=g).float()


POWERS = [10, 16, 17, 26, 33, 40, 100]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("sign,scale", [(1.0, SCALE), (-1.0, SCALE), (1.0, -SCALE)])
def test_rows(form, power, sign, scale):
    b = Batch([300, 1, 40, 0, 65], 64, 2, 16, form, seed=power)
    keys(b, scattered(power))
    q = queries(5, 6, 64, b.dtype, power, sign)
    _, out = attend(b, 6, q=q, scale=scale)
    check(out, q, b, scale, [0, 1, 2, 4])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("sign,scale", [(1.0, SCALE), (-1.0, SCALE), (1.0, -SCALE)])
def test_rows_of_prompts(form, power, sign, scale):
    b = Batch([(5 * r) % 23 for r in range(40)], 128, 1, 16, form, prompts=[500, 70], per=20, seed=power)
    keys(b, scattered(power))
    q = queries(40, 8, 128, b.dtype, power, sign)
    _, out = attend(b, 8, q=q, scale=scale)
    check(out, q, b, scale, [0, 1, 2, 3, 19, 20, 38, 39])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", [10, 17, 33, 60])
def test_parts_of_long_rows(form, power):
    """A row's keys in many parts, one key or all parts' with the largest score."""
    b = Batch([9000, 5000, 4500], 64, 1, 16, form, seed=power)
    keys(b, lambda first, n: torch.tensor([0.0 if (first + i) in (4321, 77) else -float((first + i) % 2 + 1) for i in range(n)], device="cuda"))
    q = queries(3, 4, 64, b.dtype, power)
    _, out = attend(b, 4, q=q, scale=SCALE)
    check(out, q, b, SCALE, [0, 1, 2])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", POWERS)
def test_prompts(form, power):
    b = Batch([170, 40], 64, 1, 16, form, seed=power)
    keys(b, scattered(power))
    q = queries(200, 4, 64, b.dtype, power)
    _, out, offsets = prompts(b, [160, 40], 4, q=q, scale=SCALE, behind=0)
    check(out, q, b, SCALE, [0, 1], offsets=offsets)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("steps", [2.0, -2.0])
def test_scores_that_grow_along_the_sequence(form, steps):
    """By a factor of 2^14 in weight from one 32 tokens to the next: sums are scaled anew in each tile, or never."""
    half = lambda first, n: torch.arange(first, first + n, device="cuda").div(2, rounding_mode="floor").float()  # noqa: E731
    b = Batch([(5 * r) % 23 for r in range(40)], 128, 1, 16, form, prompts=[500, 70], per=20, seed=1)
    keys(b, half)
    q = queries(40, 8, 128, b.dtype, 4, steps=steps)
    _, out = attend(b, 8, q=q, scale=SCALE)
    check(out, q, b, SCALE, [0, 1, 2, 3, 19, 20, 38, 39])
    b = Batch([400, 40], 64, 1, 16, form, seed=2)
    keys(b, half)
    q = queries(340, 4, 64, b.dtype, 4, steps=steps)
    _, out, offsets = prompts(b, [300, 40], 4, q=q, scale=SCALE, behind=0)
    check(out, q, b, SCALE, [0, 1], offsets=offsets)
