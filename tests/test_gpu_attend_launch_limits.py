"""The cache's and the attention's largest launches: 2^24 - 1 work-groups of 256 threads, which are counted in 32 bits."""
import pytest
import torch

from attend_util import attention
from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu

MOST = 2 ** 24 - 1


@pytest.fixture(autouse=True)
def memory_given_back():
    yield
    torch.cuda.empty_cache()


def refused(call):
    with pytest.raises(B.ArithSamplingError, match="one launch") as e:
        call()
    assert e.value.code == 2


def cache(kv_heads, page, dim=8, pages=1):
    g = torch.Generator(device="cuda").manual_seed(1)
    return B.Cache(*(torch.randn(pages, kv_heads, page, dim, device="cuda", generator=g).bfloat16() for _ in range(2)))


def check(c, q, out, n, heads):
    """One row's tokens are the first n of page 0."""
    k, v = (t[0, :, :n].double() for t in c._tensors)
    want, far = attention(q.view(heads, -1), k, v, torch.ones(n, dtype=torch.bool, device="cuda"), (q.numel() // heads) ** -0.5)
    assert bool(((out.view(heads, -1).double() - want).abs() <= far).all())


def test_rows():
    """16 key heads each of 2^20 rows less one; one row more is refused."""
    rows, heads = 2 ** 20 - 1, 16
    c = cache(heads, 512)
    lens = torch.full((rows + 1,), 3, dtype=torch.int32, device="cuda")
    lens[rows - 1], lens[0] = 40, 0
    table = torch.zeros(rows + 1, 1, dtype=torch.int32, device="cuda")
    q, out = (torch.randn(rows + 1, heads * 8, device="cuda").bfloat16() for _ in range(2))
    ctx = B.Ctx(rows + 1, 100)
    assert rows * heads <= MOST < (rows + 1) * heads
    refused(lambda: B.as_attend(ctx, c, B.Sequences(rows + 1, table, lens), q, out))
    last = out[rows].clone()
    B.as_attend(ctx, c, B.Sequences(rows, table, lens), q, out)
    assert torch.equal(out[rows], last) and bool((out[0] == 0).all())
    for r, n in ((1, 3), (12345, 3), (rows - 2, 3), (rows - 1, 40)):
        check(c, q[r], out[r], n, heads)


def test_many_short_rows_of_a_wave_each():
    """More rows than work-groups: four of them share one."""
    rows = 2 ** 25
    c = cache(1, 16)
    lens = (torch.arange(rows, device="cuda") % 16 + 1).int()
    table = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    q, out = (torch.randn(rows, 8, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    B.as_attend(B.Ctx(rows, 100), c, B.Sequences(rows, table, lens), q, out)
    for r in (0, 1, 2 ** 24, 2 ** 24 + 5, rows - 1):
        check(c, q[r], out[r], r % 16 + 1, 1)


def test_parts_to_join():
    """2^26 heads of queries whose prompt's part and own are joined, four to a work-group."""
    rows, heads = 2 ** 16, 1024
    c = cache(1, 16)
    lens = torch.ones(rows, dtype=torch.int32, device="cuda")
    table = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    q = torch.zeros(rows, heads * 8, device="cuda", dtype=torch.bfloat16)
    refused(lambda: B.as_attend(B.Ctx(rows, 100), c, B.Sequences(rows, table, lens, table[:1], lens[:1], rows), q, q.clone()))


def test_sequences():
    """Nearly all of them without a token."""
    rows = MOST
    c = cache(1, 16, pages=4)
    lens = torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    table = torch.zeros(rows + 1, 1, dtype=torch.int32, device="cuda")
    offsets = torch.zeros(rows + 2, dtype=torch.int64, device="cuda")
    offsets[5:] = 1
    offsets[rows:] = 3
    lens[4], lens[rows - 1] = 7, 9
    table[4], table[rows - 1] = 1, 2
    q = torch.randn(3, 8, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    ctx = B.Ctx(rows + 1, 100)
    k, v = c._tensors
    want = [t.clone() for t in (k, v)]
    refused(lambda: B.as_cache_add(ctx, c, B.Sequences(rows + 1, table, lens), q, q, offsets))
    refused(lambda: B.as_attend_prompts(ctx, c, B.Sequences(rows + 1, table, lens), q, offsets, out))
    seqs = B.Sequences(rows, table, lens)
    B.as_cache_add(ctx, c, seqs, q, q, offsets)
    for t in want:
        t[1, 0, 6], t[2, 0, 7], t[2, 0, 8] = q[0], q[1], q[2]
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    B.as_attend_prompts(ctx, c, seqs, q, offsets, out)
    for i, (page, n) in enumerate(((1, 7), (2, 8), (2, 9))):
        w, far = attention(q[i].view(1, 8), k[page].double(), v[page].double(), torch.arange(16, device="cuda") < n, 8 ** -0.5)
        assert bool(((out[i].view(1, 8).double() - w).abs() <= far).all())
