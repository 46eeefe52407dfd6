"""Each form of the attention at what single rows do not bring it to: steep, flat and turned scores of shared prompts and of ragged ones, prompts
whose rows have all ended, far pages and rows; and new tokens by offsets that are not in order."""
import pytest
import torch

from attend_util import Batch, check
from paper_2210_15458_amd import binding as B
from test_gpu_attend import FORMS, run as attend
from test_gpu_attend_prompts import run as prompts
from test_gpu_cache_add import expected, filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("gain,scale", [(60.0, 1.0), (60.0, -1.0), (1.0, 0.0), (1.0, -0.3)])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (256, 16), (72, 8)])
def test_steep_flat_and_turned_scores(form, gain, scale, dim, page):
    b = Batch([(3 * r) % 20 for r in range(40)], dim, 1, page, form, prompts=[300, 90], per=20, seed=4)
    q, out = attend(b, 8, gain=gain, scale=scale)
    check(out, q, b, scale=scale, rows=[0, 1, 7, 19, 20, 39])
    b = Batch([260, 30], dim, 1, page, form, seed=5)
    q = (gain * torch.randn(230, 4 * dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))).to(b.dtype)
    _, out, _ = prompts(b, [200, 30], 4, q=q, scale=scale, behind=0)
    check(out[170:], q[170:], b, scale=scale, offsets=[0, 30, 60])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
@pytest.mark.parametrize("own", [True, False])
def test_prompts_whose_rows_have_all_ended(form, window, sinks, own):
    lens = [(3 * r) % 20 if own else 0 for r in range(80)]
    b = Batch(lens, 64, 2, 16, form, prompts=[300, 200, 90, 130], per=20, seed=7)
    if not own:
        b.table = b.lens = None
    finished = torch.zeros(80, dtype=torch.uint8, device="cuda")
    finished[20:40], finished[60:79] = 1, 3
    q, out = attend(b, 8, window=window, sinks=sinks, finished=finished)
    assert bool((out[20:40] == 7).all()) and bool((out[60:79] == 7).all())
    check(out, q, b, window=window, sinks=sinks, rows=[0, 1, 19, 40, 59, 79])
    finished[:] = 1
    _, out = attend(b, 8, window=window, sinks=sinks, finished=finished, q=q)
    assert bool((out == 7).all())


def test_far_pages_and_rows_by_128_queries():
    """A cache of more than 2^32 values, a prompt and rows in its last pages; rows of q and out more than 2^31 values from the first."""
    dim, page, rows = 64, 16, 40
    pages = (1 << 32) // (page * dim) + 64
    b = Batch([(3 * r) % 9 + 1 for r in range(rows)], dim, 1, page, "bf16 128", prompts=[200], per=rows, seed=1)
    k, v = (torch.zeros(pages, 1, page, dim, dtype=b.dtype, device="cuda") for _ in range(2))
    shift = pages - b.k.shape[0]
    k[shift:], v[shift:] = b.k, b.v
    apart = (1 << 31) // (rows - 1) + 8
    wide = torch.empty(apart * rows, dtype=b.dtype, device="cuda")
    q = wide.as_strided((rows, 512), (apart, 1))
    out = q[:, 256:]
    q[:, :256].normal_()
    ctx = B.Ctx(rows, 100)
    ctx.set_tuning("attend_shape", 2)
    B.as_attend(ctx, B.Cache(k, v), B.Sequences(rows, b.table + shift, b.lens, b.prompt_table + shift, b.prompt_lens, rows), q[:, :256], out)
    check(out, q[:, :256], b, rows=[0, 1, 20, rows - 1])
    x, y = q[:, :256], torch.zeros(rows, 256, dtype=b.dtype, device="cuda")
    alone = Batch([150], dim, 1, page, "bf16 128", seed=2)
    shift = pages - alone.k.shape[0]
    k[shift:], v[shift:] = alone.k, alone.v
    B.as_attend_prompts(ctx, B.Cache(k, v), B.Sequences(1, alone.table + shift, alone.lens), x, torch.tensor([0, rows], device="cuda"), y)
    check(y, x, alone, offsets=[0, rows])


@pytest.mark.parametrize("offsets,taken", [([-100, 20, 1 << 40], [0, 20, 50]), ([-3, -2, 50], [0, 0, 50]), ([7, 20, 20], [7, 20, 20]), ([60, 70, 80], [50, 50, 50])])
def test_offsets_beyond_the_tokens_are_held_at_their_ends(offsets, taken):
    k, v = filled((11, 1, 16, 64), torch.bfloat16, 1), filled((11, 1, 16, 64), torch.bfloat16, 2)
    table, lens = torch.tensor([[3, 9, 0, 5], [10, 1, 7, 2]], dtype=torch.int32), [60, 64]
    new = filled((50, 64), torch.bfloat16, 3)
    want = [expected(c, table.tolist(), lens, new.view(50, 1, 64), taken, 16) for c in (k, v)]
    B.as_cache_add(B.Ctx(50, 100), B.Cache(k, v), B.Sequences(2, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")), new, new,
                   torch.tensor(offsets, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("offsets", [[50, 0, 50], [1 << 50, -(1 << 50), 7], [20, 50, 3]])
def test_offsets_that_fall_leave_pages_of_nobody_alone(offsets):
    k, v = filled((11, 1, 16, 64), torch.bfloat16, 1), filled((11, 1, 16, 64), torch.bfloat16, 2)
    before = [t[[4, 6, 8]].clone() for t in (k, v)]
    table = torch.tensor([[3, 9, 0, 5], [10, 1, 7, 2]], dtype=torch.int32, device="cuda")
    new = filled((50, 64), torch.bfloat16, 3)
    B.as_cache_add(B.Ctx(50, 100), B.Cache(k, v), B.Sequences(2, table, torch.tensor([60, 64], dtype=torch.int32, device="cuda")), new, new,
                   torch.tensor(offsets, device="cuda"))
    torch.cuda.synchronize()
    assert all(torch.equal(t[[4, 6, 8]], b) for t, b in zip((k, v), before))
