"""Attention of one query a row over a paged cache (as_attend): against its definition in 64 bits, in caches whose unused slots hold
NaN and whose tables name no pages past a length."""
import pytest
import torch

from attend_util import NAN, Batch, check
from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu

FORMS = ["bf16", "bf16 16", "bf16 128", "f32"]     # (the last number: queries of a work-group, whatever the rule would have)


def run(batch, heads, window=0, sinks=0, scale=None, finished=None, pad=0, ctx=None, seed=5, gain=1.5, q=None):
    rows, dim = len(batch.own), batch.dim
    g = torch.Generator(device="cuda").manual_seed(seed)
    if q is None:
        wide = (gain * torch.randn(rows, heads * dim + pad, device="cuda", generator=g)).to(batch.dtype)
        q = wide[:, pad // 2:pad // 2 + heads * dim]
    out = torch.full((rows, heads * dim + pad), 7.0, dtype=batch.dtype, device="cuda")
    ctx = ctx or B.Ctx(max(rows, 1), 100, torch.float32)
    if batch.shape:
        ctx.set_tuning("attend_shape", batch.shape)
    seqs = B.Sequences(rows, batch.table, batch.lens, batch.prompt_table, batch.prompt_lens, batch.per, finished)
    B.as_attend(ctx, B.Cache(batch.k, batch.v), seqs, q, out[:, pad // 2:pad // 2 + heads * dim], scale=scale, window=window, sinks=sinks)
    torch.cuda.synchronize()
    if pad:
        assert bool((out[:, :pad // 2] == 7).all()) and bool((out[:, pad // 2 + heads * dim:] == 7).all())
    return q, out[:, pad // 2:pad // 2 + heads * dim]


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("dim,kv_heads,group,page", [(64, 2, 4, 16), (128, 1, 1, 16), (128, 3, 8, 64), (256, 2, 2, 16), (8, 1, 3, 4), (72, 2, 5, 1),
                                                     (136, 1, 16, 8), (96, 2, 17, 32), (128, 1, 33, 2), (200, 1, 4, 128), (192, 1, 4, 16), (104, 2, 2, 16), (64, 5, 1, 1024)])
def test_lengths(dtype, dim, kv_heads, group, page):
    own = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 130, 257, 300]
    b = Batch(own, dim, kv_heads, page, dtype, seed=dim + group)
    q, out = run(b, kv_heads * group, pad=6)
    print("worst", check(out, q, b))


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("dim,group,page,window,sinks", [(64, 2, 16, 1, 0), (128, 4, 16, 5, 1), (128, 1, 4, 32, 0), (72, 3, 16, 33, 40), (64, 8, 32, 100, 7),
                                                         (256, 2, 64, 64, 64), (128, 4, 16, 1000, 3), (64, 1, 16, 2147483647, 2147483647)])
def test_windows_and_first_tokens(dtype, dim, group, page, window, sinks):
    own = [0, 1, 5, 6, 31, 33, 64, 99, 100, 101, 107, 150, 290]
    b = Batch(own, dim, 2, page, dtype, seed=window % 1000)
    for r, n in enumerate(own):                   # what the window hides may be anything
        for t in range(sinks, max(n - window, 0)):
            p, i = b.place(r, t)
            b.k[p, :, i] = NAN
            b.v[p, :, i] = float("inf") if t % 2 else NAN
    q, out = run(b, 2 * group, window=window, sinks=sinks)
    print("worst", check(out, q, b, window=window, sinks=sinks))


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("dim,kv_heads,group,page,per", [(64, 2, 4, 16, 4), (128, 1, 1, 16, 33), (72, 2, 3, 8, 5), (128, 2, 8, 64, 16), (256, 1, 2, 16, 70)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3), (7, 200)])
def test_prompts_shared_by_rows(dtype, dim, kv_heads, group, page, per, window, sinks):
    prompts = [0, 1, 130, 64, 300]
    rows = per * len(prompts) - (per > 4)          # (the last prompt one row short)
    own = [(7 * r) % 45 for r in range(rows)]
    b = Batch(own, dim, kv_heads, page, dtype, prompts=prompts, per=per, seed=per)
    q, out = run(b, kv_heads * group, window=window, sinks=sinks)
    rows = sorted({0, 1, per, per + 1, 2 * per, 2 * per + 1, 3 * per - 1, 3 * per, 4 * per, 4 * per + 1, rows - 1})
    print("worst", check(out, q, b, window=window, sinks=sinks, rows=rows))


@pytest.mark.parametrize("dtype", FORMS)
def test_prompts_alone_and_split(dtype):
    """No tokens of the rows' own; one row over a long prompt, whose keys are split and joined."""
    b = Batch([0, 0], 128, 2, 16, dtype, prompts=[5000], per=2, seed=3)
    b.table = b.lens = None
    q, out = run(b, 8)
    print("worst", check(out, q, b))


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 0), (1500, 2000), (20000, 5)])
def test_long_split(dtype, window, sinks):
    b = Batch([9000, 1, 4097, 0, 12345], 64, 1, 16, dtype, seed=9, room=2000)
    q, out = run(b, 3, window=window, sinks=sinks)
    print("worst", check(out, q, b, window=window, sinks=sinks))


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("prompts", [None, [100, 20]])
def test_finished_rows_are_left_as_they_were(dtype, prompts):
    own = [40, 3, 0, 700, 64, 9]
    b = Batch(own, 64, 2, 16, dtype, prompts=prompts, per=3)
    finished = torch.tensor([0, 1, 0, 0, 255, 1], dtype=torch.uint8, device="cuda")
    q, out = run(b, 4, finished=finished)
    assert bool((out[[1, 4, 5]] == 7).all())
    check(out, q, b, rows=[0, 2, 3])


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("per", [3, 40])
def test_no_numbers_reach_those_that_see_them_only(dtype, per):
    """A value of the prompt that is infinite or NaN, in the window of some rows and not of others; a NaN in one row's query."""
    own = [(5 * r) % 11 for r in range(2 * per)]
    b = Batch(own, 64, 2, 16, dtype, prompts=[90, 70], per=per, seed=1)
    window = 12
    marks = {(0, 83): float("inf"), (0, 85): NAN, (0, 3): NAN, (per, 62): -float("inf")}
    for (r, t), x in marks.items():
        p, i = b.place(r, t)
        b.v[p, 1, i, t % 64] = x
        b.k[p, 0, i] = b.k[p, 0, i]
    clean = b.v.clone()
    clean[~clean.isfinite()] = 0
    rows = 2 * per
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(rows, 6 * 64, device="cuda", generator=g).to(b.dtype)
    q[1, 70] = NAN                               # row 1, head 1: its key head is 0
    _, out = run(b, 6, window=window, sinks=2, q=q)
    marked = b.v
    for r in range(rows):
        total = b.prompts[r // per] + own[r]
        got = out[r].view(6, 64)
        hit = {t: x for (first, t), x in marks.items() if first // per == r // per and (t > total - 1 - window)}
        for h in range(6):
            if r == 1 and h == 1:
                assert bool(got[h].isnan().all())
                continue
            odd = {t % 64: x for t, x in hit.items()} if h >= 3 else {}
            for d in range(64):
                if d in odd and odd[d] != odd[d]:
                    assert bool(got[h, d].isnan())
                elif d in odd:
                    assert float(got[h, d]) == odd[d]
                else:
                    assert bool(got[h, d].isfinite()), (r, h, d)
    # and where there is a number it is the right one
    b.v = torch.where(marked.isfinite() | marked.isnan() & clean.isnan(), marked, clean)
    q2, out2 = run(b, 6, window=window, sinks=2, q=torch.where(q.isnan(), torch.zeros_like(q), q))
    same = out.isfinite()
    assert torch.equal(out[same], out2[same])
    check(out2, q2, b, window=window, sinks=2, rows=[0, 1, per, rows - 1])


def test_steep_and_flat_scores():
    """Scores far beyond what an exponential without a maximum taken off could hold, and all alike."""
    for dtype in FORMS:
        b = Batch([200, 77], 64, 1, 16, dtype, seed=4)
        q, out = run(b, 2, gain=60.0, scale=1.0)
        check(out, q, b, scale=1.0)
        q, out = run(b, 2, scale=0.0)
        check(out, q, b, scale=0.0)
        q, out = run(b, 2, scale=-0.3)
        check(out, q, b, scale=-0.3)


def test_lengths_beyond_the_table_and_below_zero():
    b = Batch([64, 32, 48], 64, 1, 16, "bf16", seed=6)
    b.lens[0], b.lens[1] = 1000, -3
    q, out = run(b, 2)
    assert bool((out[1] == 0).all())
    check(out, q, b, rows=[0, 2])


def test_pages_that_are_not_there_are_not_followed():
    """An entry outside [0, pages) inside a length: some page is read, nothing outside the cache, and other rows are right."""
    b = Batch([64, 33, 48], 64, 1, 16, "bf16", seed=6)
    b.table[1, 0], b.table[1, 1] = -5, 1 << 30
    q, out = run(b, 2)
    check(out, q, b, rows=[0, 2])


def test_same_bits_each_time_and_whatever_the_other_rows_are():
    b = Batch([3000, 17, 900], 128, 2, 16, "bf16", prompts=[600, 40, 5], per=1, seed=8)
    q, one = run(b, 8)
    _, two = run(b, 8, q=q)
    assert torch.equal(one, two)
    other = q.clone()
    other[0] = NAN
    _, three = run(b, 8, q=other)
    assert torch.equal(one[1:], three[1:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,kv_heads,group,page,room", [(64, 3, 4, 16, 64), (128, 8, 4, 16, 200), (72, 3, 3, 8, 90), (96, 2, 1, 16, 40), (256, 3, 2, 64, 300), (192, 2, 5, 1, 33),
                                                          (128, 4, 20, 16, 500)])
@pytest.mark.parametrize("prompts", [False, True])
def test_many_short_rows(dtype, dim, kv_heads, group, page, room, prompts):
    """So many that each is one wave's, with what its prompt left and without; some finished, some empty."""
    rows = -(-2048 // kv_heads // 10) * 10 + 10
    own = [(r * 37) % (room + 1) for r in range(rows)]
    own[3] = room
    b = Batch(own, dim, kv_heads, page, dtype, prompts=[0, 33, 70][:2] + [5] * (rows // 10 - 2) if prompts else None, per=10, seed=dim)
    assert rows * kv_heads >= 2048 and b.table.shape[1] * page <= 512
    finished = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    finished[7], finished[rows - 2] = 1, 1
    keep = [0, 1, 2, 3, 11, 12, 19, 20, 55, rows // 2, rows - 1]
    for window, sinks in ((0, 0), (11, 3)):
        q, out = run(b, kv_heads * group, window=window, sinks=sinks, finished=finished, pad=2)
        assert bool((out[[7, rows - 2]] == 7).all())
        check(out, q, b, window=window, sinks=sinks, rows=keep)


@pytest.mark.parametrize("dtype", FORMS)
def test_a_thousand_heads_on_one(dtype):
    b = Batch([70, 3], 8, 1, 16, dtype, prompts=[40], per=2, seed=7)
    q, out = run(b, 1024)
    check(out, q, b)
