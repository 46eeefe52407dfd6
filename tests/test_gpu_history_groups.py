"""as_history_set where several rows of a prompt share a block, which marks the prompt's tokens once for all of them: with whole
and ragged last groups, rows left out, short and long lists; exactly."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_shaping import history64, pack

pytestmark = pytest.mark.gpu


def record(rows, V):
    return (torch.zeros(rows, (V + 31) // 32, dtype=torch.int32, device="cuda"), torch.zeros(rows, V, dtype=torch.int32, device="cuda"))


def own_tokens(rng, rows, V, T):
    """Tokens that no two rows share: row r has only such as are r modulo the number of rows."""
    return (rng.integers(0, V // rows, (rows, T)) * rows + np.arange(rows)[:, None]).astype(np.int32)


def ragged(rng, prompts, P, V):
    lens = rng.integers(P // 2, P + 1, prompts)
    offsets = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    return rng.integers(0, V, max(1, offsets[-1])).astype(np.int32), offsets


def dev(a):
    return torch.from_numpy(a).cuda()


# rows a block: 4, of 67 (17 groups, the last of 3); 18 with lists beyond 4096 tokens (4 groups, the last of 13); 4 of 64;
# 2 of 16; rows that are no whole number of prompts
@pytest.mark.parametrize("rows,per,V,P,T", [(536, 67, 70001, 60, 40), (536, 67, 70001, 6000, 40), (1024, 64, 32128, 512, 64),
                                            (16, 16, 256000, 9000, 4096), (500, 67, 70001, 300, 0), (530, 67, 70001, 0, 33)])
def test_rows_that_share_a_block(rows, per, V, P, T):
    prompts = (rows + per - 1) // per
    rng = np.random.default_rng(rows + P)
    ctx = B.Ctx(rows, V, torch.float32)
    seen, counts = record(rows, V)
    want_seen, want_counts = None, None
    for turn in range(3):                    # over what the turn before has left; in the last two some rows are left alone
        pt, offsets = ragged(rng, prompts, P, V)
        tt = own_tokens(rng, rows, V, T)
        lens = rng.integers(0, T + 1, rows).astype(np.int32)
        which = np.ones(rows, dtype=np.uint8) if turn == 0 else (rng.random(rows) < 0.7).astype(np.uint8)
        if turn == 2:
            which[::per] = 0                 # the first row of each prompt among them, and a whole prompt
            which[:per] = 0
        print(f"rows {rows} of {per}, V {V}, lists {P} + {T}, turn {turn}", flush=True)
        B.as_history_set(ctx, seen, counts, dev(pt), dev(offsets), per, dev(tt) if T else None, dev(lens) if T else None,
                         which=None if turn == 0 else dev(which))
        s, c = history64(rows, V, pt, offsets, per, tt if T else None, lens)
        live = which.astype(bool)[:, None]
        want_seen = s if want_seen is None else np.where(live, s, want_seen)
        want_counts = c if want_counts is None else np.where(live, c, want_counts)
        assert torch.equal(seen, pack(want_seen)), turn
        assert torch.equal(counts, dev(want_counts)), turn


@pytest.mark.parametrize("rows,V", [(16, 32128), (600, 70001)])
@pytest.mark.parametrize("past", [1, 1000, 2 ** 31 - 1])
def test_rows_per_prompt_beyond_the_rows(rows, V, past):
    """One prompt for all, said as a number of rows that there are not: the rows that are there are all that is worked on."""
    per = past if past > rows else rows + past
    rng = np.random.default_rng(rows)
    seen, counts = record(rows, V)
    pt, offsets = ragged(rng, 1, 4000, V)
    tt = own_tokens(rng, rows, V, 25)
    print(f"rows {rows} of {per}, V {V}", flush=True)
    B.as_history_set(B.Ctx(rows, V, torch.float32), seen, counts, dev(pt), dev(offsets), per, dev(tt))
    want_seen, want_counts = history64(rows, V, pt, offsets, per, tt, np.full(rows, 25))
    assert torch.equal(seen, pack(want_seen)) and torch.equal(counts, dev(want_counts))


def test_the_context_s_vocabulary():
    """Tokens past the context's vocabulary are left out, whatever the buffers have room for; a layer does not look at it."""
    rows, V, room = 5, 100, 1000
    seen, counts = record(rows, room)
    ctx = B.Ctx(rows, V, torch.float32)
    tt = dev(np.tile(np.array([[3, 99, 100, 999]], dtype=np.int32), (rows, 1)))
    B.as_history_set(ctx, seen, counts, tokens=tt)
    B.as_history_add(ctx, seen, counts, torch.full((rows,), 500, dtype=torch.int32, device="cuda"))
    want = np.zeros((rows, room), dtype=np.int32)
    want[:, [3, 99]] = 1
    assert torch.equal(counts, dev(want)) and torch.equal(seen, pack(want > 0))
    out = torch.empty(rows, room, device="cuda")
    B.as_linear(ctx, B.Layer(torch.ones(room, 8, device="cuda")), torch.ones(rows, 8, device="cuda"), out)
    assert bool((out == 8.0).all())
