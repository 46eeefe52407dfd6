"""New tokens into a paged cache (as_cache_add): every slot of the cache, bit for bit."""
import pytest
import torch

from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu


def filled(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, device="cuda", generator=g).to(dtype)


def expected(cache, table, lens, new, offsets, page, finished=None):
    """new: [tokens, kv_heads, dim]."""
    want = cache.clone()
    pages = cache.shape[0]
    for s, n in enumerate(lens):
        a, b = offsets[s], offsets[s + 1]
        if finished is not None and finished[s]:
            continue
        for t in range(a, b):
            pos = n - (b - t)
            if 0 <= pos < len(table[s]) * page and 0 <= table[s][pos // page] < pages:
                want[table[s][pos // page], :, pos % page] = new[t]
    return want


def tables(rows, width, pages, seed):
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:rows * width]
    return order.view(rows, width).int()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,kv_heads,page", [(64, 2, 16), (128, 8, 16), (8, 1, 1), (72, 3, 4), (256, 5, 64), (200, 1, 2), (64, 33, 8)])
@pytest.mark.parametrize("pad", [0, 5])
def test_one_token_a_row(dtype, dim, kv_heads, page, pad):
    rows, width = 37, 3
    k, v = filled((rows * width + 2, kv_heads, page, dim), dtype, 1), filled((rows * width + 2, kv_heads, page, dim), dtype, 2)
    table = tables(rows, width, rows * width + 2, 3)
    lens = [(i * 5) % (width * page) + 1 for i in range(rows)]
    lens[3], lens[4], lens[5] = 0, -4, width * page + 1          # (no place for their tokens)
    table[6] = torch.tensor([-1, 1 << 30, -9])
    new = filled((rows, 2 * kv_heads * dim + pad), dtype, 4)
    nk, nv = new[:, pad // 2:pad // 2 + kv_heads * dim], new[:, pad // 2 + kv_heads * dim:pad // 2 + 2 * kv_heads * dim]
    finished = torch.zeros(rows, dtype=torch.uint8)
    finished[[0, 9, 36]] = torch.tensor([1, 255, 4], dtype=torch.uint8)
    want = [expected(c, table.tolist(), lens, x.reshape(rows, kv_heads, dim), list(range(rows + 1)), page, finished.tolist()) for c, x in ((k, nk), (v, nv))]
    seqs = B.Sequences(rows, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), finished=finished.cuda())
    B.as_cache_add(B.Ctx(rows, 100), B.Cache(k, v), seqs, nk, nv)
    torch.cuda.synchronize()
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,kv_heads,page", [(64, 2, 16), (128, 8, 16), (8, 1, 1), (72, 3, 4), (256, 5, 64)])
def test_ragged(dtype, dim, kv_heads, page):
    new = [0, 1, 70, 0, 33, 5, 0, 129, 2]
    had = [3, 0, 9, 0, 40, 100, 7, 1, 63]
    rows, room = len(new), 192
    width = -(-room // page)
    lens = [a + n for a, n in zip(had, new)]
    lens[5] = 2                                                   # (three of its five have no place)
    before, behind = 2, 4
    offsets = [before]
    for n in new:
        offsets.append(offsets[-1] + n)
    total = offsets[-1] + behind
    k, v = filled((rows * width + 1, kv_heads, page, dim), dtype, 1), filled((rows * width + 1, kv_heads, page, dim), dtype, 2)
    table = tables(rows, width, rows * width + 1, 3)
    nk, nv = filled((total, kv_heads, dim), dtype, 5), filled((total, kv_heads, dim), dtype, 6)
    finished = torch.zeros(rows, dtype=torch.uint8)
    finished[4] = 1
    want = [expected(c, table.tolist(), lens, x, offsets, page, finished.tolist()) for c, x in ((k, nk), (v, nv))]
    seqs = B.Sequences(rows, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), finished=finished.cuda())
    B.as_cache_add(B.Ctx(total, 100), B.Cache(k, v), seqs, nk, nv, torch.tensor(offsets, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_pages_apart():
    """One layer's pages inside a larger tensor: nothing between them changes."""
    both = filled((7, 3, 2, 16, 64), torch.bfloat16, 1)
    k, v = both[:, 0], both[:, 2]
    table = torch.tensor([[4, 1], [6, 2]], dtype=torch.int32, device="cuda")
    new = filled((2, 2 * 64), torch.bfloat16, 3)
    want = both.clone()
    want[1, 0, :, 3], want[6, 0, :, 15] = new[0].view(2, 64), new[1].view(2, 64)
    want[1, 2, :, 3], want[6, 2, :, 15] = new[0].view(2, 64), new[1].view(2, 64)
    seqs = B.Sequences(2, table, torch.tensor([20, 16], dtype=torch.int32, device="cuda"))
    B.as_cache_add(B.Ctx(2, 100), B.Cache(k, v), seqs, new, new)
    torch.cuda.synchronize()
    assert torch.equal(both, want)


def test_offsets_out_of_range_are_not_followed():
    k, v = filled((8, 1, 16, 64), torch.bfloat16, 1), filled((8, 1, 16, 64), torch.bfloat16, 2)
    table = tables(2, 4, 8, 1).cuda()
    seqs = B.Sequences(2, table, torch.tensor([60, 64], dtype=torch.int32, device="cuda"))
    new = filled((50, 64), torch.bfloat16, 3)
    for offsets in ([-100, 20, 1 << 40], [50, 0, 50], [1 << 50, -(1 << 50), 7]):
        B.as_cache_add(B.Ctx(50, 100), B.Cache(k, v), seqs, new, new, torch.tensor(offsets, device="cuda"))
    torch.cuda.synchronize()
