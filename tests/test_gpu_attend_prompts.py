"""Attention of ragged prompts over a paged cache (as_attend_prompts): against its definition in 64 bits, in caches whose unused slots
hold NaN and whose tables name no pages past a length."""
import pytest
import torch

from attend_util import NAN, Batch, check
from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu

FORMS = ["bf16", "bf16 16", "bf16 128", "f32"]     # (the last number: queries of a work-group, whatever the rule would have)


def run(batch, new, heads, window=0, sinks=0, finished=None, pad=0, before=0, behind=3, seed=5, q=None, ctx=None, scale=None):
    """new: queries of each row; before, behind: rows of q and out that are nobody's."""
    dim, n = batch.dim, before + sum(new) + behind
    g = torch.Generator(device="cuda").manual_seed(seed)
    if q is None:
        q = (1.5 * torch.randn(n, heads * dim + pad, device="cuda", generator=g)).to(batch.dtype)[:, pad // 2:pad // 2 + heads * dim]
    offsets = [before]
    for x in new:
        offsets.append(offsets[-1] + x)
    out = torch.full((n, heads * dim + pad), 7.0, dtype=batch.dtype, device="cuda")
    ctx = ctx or B.Ctx(max(n, len(new)), 100, torch.float32)
    if batch.shape:
        ctx.set_tuning("attend_shape", batch.shape)
    seqs = B.Sequences(len(new), batch.table, batch.lens, finished=finished)
    B.as_attend_prompts(ctx, B.Cache(batch.k, batch.v), seqs, q, torch.tensor(offsets, device="cuda"), out[:, pad // 2:pad // 2 + heads * dim],
                        window=window, sinks=sinks, scale=scale)
    torch.cuda.synchronize()
    assert bool((out[:before] == 7).all()) and bool((out[n - behind:] == 7).all() if behind else True), "rows that are nobody's"
    if pad:
        assert bool((out[:, :pad // 2] == 7).all()) and bool((out[:, pad // 2 + heads * dim:] == 7).all())
    return q, out[:, pad // 2:pad // 2 + heads * dim], offsets


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("dim,kv_heads,group,page", [(64, 2, 4, 16), (128, 1, 1, 16), (128, 2, 8, 64), (256, 1, 2, 16), (8, 1, 3, 4), (72, 2, 5, 1),
                                                     (136, 1, 16, 8), (96, 1, 17, 32), (200, 1, 4, 128), (192, 1, 4, 16), (104, 2, 2, 16), (64, 3, 1, 1024)])
def test_chunks(dtype, dim, kv_heads, group, page):
    new = [1, 0, 3, 33, 64, 0, 0, 17, 130, 1]
    had = [0, 5, 70, 0, 31, 0, 9, 200, 33, 299]
    b = Batch([a + n for a, n in zip(had, new)], dim, kv_heads, page, dtype, seed=dim)
    q, out, offsets = run(b, new, kv_heads * group, pad=10, before=2)
    print("worst", check(out, q, b, offsets=offsets))


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("dim,group,page,window,sinks", [(64, 2, 16, 1, 0), (128, 4, 16, 5, 1), (128, 1, 4, 32, 0), (72, 3, 16, 33, 40), (64, 8, 32, 100, 7),
                                                         (256, 2, 64, 64, 64), (128, 4, 16, 1000, 3), (128, 2, 16, 129, 100)])
def test_windows_and_first_tokens(dtype, dim, group, page, window, sinks):
    new, had = [150, 1, 40, 200, 9], [0, 290, 131, 64, 0]
    b = Batch([a + n for a, n in zip(had, new)], dim, 1, page, dtype, seed=window)
    for r, (a, n) in enumerate(zip(had, new)):    # what the window hides from all queries of a row
        for t in range(sinks, max(a - window + 1, 0)):
            p, i = b.place(r, t)
            b.k[p, :, i] = NAN
            b.v[p, :, i] = float("inf") if t % 2 else NAN
    q, out, offsets = run(b, new, group, window=window, sinks=sinks)
    print("worst", check(out, q, b, window=window, sinks=sinks, offsets=offsets))


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("had,new", [(0, 700), (6000, 5), (3000, 400)])
def test_long(dtype, had, new):
    b = Batch([had + new, 3], 128, 2, 16, dtype, seed=had, room=700)
    q, out, offsets = run(b, [new, 3], 4)
    keep = list(range(0, new, 37)) + [new - 1]
    full = [torch.cat([x[keep], x[new:new + 3]]) for x in (q, out)]
    # (some of the row's queries, each as if it were the last of the row)
    for j, i in enumerate(keep):
        check(full[1][j:j + 1], full[0][j:j + 1], Shorter(b, had + i + 1), rows=[0], offsets=[0, 1])
    check(out, q, b, rows=[1], offsets=offsets)


class Shorter:
    """Row 0 of a batch, cut behind its first n tokens."""

    def __init__(self, batch, n):
        self.batch, self.n, self.dim, self.own = batch, n, batch.dim, batch.own

    def tokens(self, r):
        return [x[:, :self.n] for x in self.batch.tokens(r)]


@pytest.mark.parametrize("dtype", FORMS)
def test_no_numbers_of_later_tokens_stay_there(dtype):
    """A token whose value is infinite or NaN: queries before it do not see it, those behind it do until a window leaves it."""
    for window, sinks in ((0, 0), (20, 0), (20, 3)):
        n, heads, dim = 150, 2, 64
        b = Batch([n], dim, 1, 16, dtype, seed=2)
        marks = {40: float("inf"), 100: NAN, 1: -float("inf")}
        for t, x in marks.items():
            p, i = b.place(0, t)
            b.v[p, 0, i, t % dim] = x
        q, out, _ = run(b, [n], heads, window=window, sinks=sinks)
        for i in range(n):
            got = out[i].view(heads, dim)
            seen = {t % dim: x for t, x in marks.items() if t <= i and (window == 0 or t > i - window or t < sinks)}
            for d in range(dim):
                for h in range(heads):
                    x = seen.get(d, 0.0)
                    if x != x:
                        assert bool(got[h, d].isnan()), (i, d)
                    elif x:
                        assert float(got[h, d]) == x, (i, d)
                    else:
                        assert bool(got[h, d].isfinite()), (i, d)
        p, i = b.place(0, 0)
        odd = ~b.v.isfinite() & ~b.v.isnan()
        clean = b.v.clone()
        clean[odd] = 0
        p, i = b.place(0, 100)
        clean[p, 0, i, 100 % dim] = 0
        b.v = clean
        q2, out2, offsets = run(b, [n], heads, window=window, sinks=sinks, q=q)
        same = out[:n].isfinite()
        assert torch.equal(out[:n][same], out2[:n][same])
        check(out2, q2, b, window=window, sinks=sinks, offsets=offsets)


@pytest.mark.parametrize("dtype", FORMS)
def test_a_query_that_is_no_number_stays_alone(dtype):
    b = Batch([100], 128, 1, 16, dtype, seed=12)
    q, out, offsets = run(b, [100], 2)
    bad = q.clone()
    bad[50, 128 + 5] = NAN
    _, other, _ = run(b, [100], 2, q=bad)
    assert bool(other[50, 128:].isnan().all())
    other[50, 128:] = out[50, 128:]
    assert torch.equal(out, other)


@pytest.mark.parametrize("long", [False, True])
def test_finished_sequences_are_left_as_they_were(long):
    new = [20, 30, 1, 9]
    had = [0, 4, 60, 5000 if long else 5]
    b = Batch([a + n for a, n in zip(had, new)], 64, 2, 16, "bf16", room=400 if long else None)
    finished = torch.tensor([0, 1, 0, 0], dtype=torch.uint8, device="cuda")
    q, out, offsets = run(b, new, 4, finished=finished)
    assert bool((out[20:50] == 7).all())
    check(out, q, b, rows=[0, 2, 3], offsets=offsets)


def test_many_sequences():
    """More than a search looks at in one step, most of them empty."""
    new = [(i * 7919) % 5 if i % 3 == 0 else 0 for i in range(5000)]
    b = Batch([n + i % 2 for i, n in enumerate(new)], 64, 1, 16, "bf16", seed=3)
    q, out, offsets = run(b, new, 3)
    rows = [r for r in range(0, 5000, 41)] + [4998, 4999]
    check(out, q, b, rows=rows, offsets=offsets)


def test_more_queries_than_tokens():
    """Queries whose positions come out below zero see nothing."""
    b = Batch([5, 8], 64, 1, 16, "bf16", seed=3)
    b.lens[0] = 5
    q, out, offsets = run(b, [9, 8], 2)
    assert bool((out[:4] == 0).all())
    check(out, q, b, rows=[1], offsets=offsets)
    check(out[4:9], q[4:9], b, rows=[0], offsets=[0, 5])


def test_offsets_out_of_range_are_not_followed():
    b = Batch([40, 30, 20], 64, 1, 16, "bf16", seed=3)
    n = 90
    q = torch.randn(n, 128, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    ctx = B.Ctx(n, 100, torch.float32)
    for offsets in ([-5, 40, 70, 1 << 40], [40, 0, 90, 20], [1 << 50, -(1 << 50), 3, 4]):
        B.as_attend_prompts(ctx, B.Cache(b.k, b.v), B.Sequences(3, b.table, b.lens), q, torch.tensor(offsets, device="cuda"), out)
    torch.cuda.synchronize()
    B.as_attend_prompts(ctx, B.Cache(b.k, b.v), B.Sequences(3, b.table, b.lens), q, torch.tensor([0, 40, 70, 90], device="cuda"), out)
    check(out, q, b, offsets=[0, 40, 70, 90])


@pytest.mark.parametrize("dtype", FORMS)
def test_a_thousand_heads_on_one(dtype):
    b = Batch([9, 40], 8, 1, 16, dtype, seed=7)
    q, out, offsets = run(b, [2, 3], 1024)
    check(out, q, b, offsets=offsets)
