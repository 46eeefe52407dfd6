"""The cache's and the attention's calls as a program makes them: refusals, streams, captures, the workspace, far offsets."""
import ctypes as C
import math

import pytest
import torch

from attend_util import Batch, check
from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu

INVALID, UNSUPPORTED, ALLOC = 1, 2, 3


def setup(rows=4, prompts=False, dtype="bf16"):
    b = Batch([40] * rows, 64, 2, 16, dtype, prompts=[30] * (rows // 2) if prompts else None, per=2)
    ctx = B.Ctx(64, 100, torch.float32)
    q = torch.randn(rows, 256, device="cuda").to(b.dtype)
    return b, ctx, B.Cache(b.k, b.v), B.Sequences(rows, b.table, b.lens, b.prompt_table, b.prompt_lens, b.per), q, torch.zeros_like(q)


def test_refusals():
    b, ctx, cache, seqs, q, out = setup()
    lib = B.lib()
    offsets = torch.tensor([0, 1, 2, 3, 4], device="cuda")

    def attend(rows=4, qp=q.data_ptr(), ldq=256, heads=4, scale=0.125, window=0, sinks=0, op=out.data_ptr(), ldo=256, s=seqs, c=cache):
        return lib.as_attend(ctx._h, c._ref, s._ref, rows, qp, ldq, heads, scale, window, sinks, op, ldo)

    def prompts(tokens=4, at=offsets.data_ptr(), s=seqs, **kw):
        return lib.as_attend_prompts(ctx._h, cache._ref, s._ref, kw.get("rows", 4), q.data_ptr(), 256, tokens, at, 4, 0.125, 0, 0, out.data_ptr(), 256)

    def add(rows=4, tokens=4, at=None, kp=q.data_ptr(), ldk=256, s=seqs):
        return lib.as_cache_add(ctx._h, cache._ref, s._ref, rows, kp, ldk, q.data_ptr(), 256, tokens, at)

    def refused(rc, *words, code=INVALID):
        text = lib.as_last_error(ctx._h).decode()
        assert rc == code and all(w in text for w in words), (rc, text)

    assert attend(rows=0) == 0 and prompts(tokens=0) == 0 and add(rows=0, tokens=0) == 0
    refused(attend(rows=65), "rows")
    refused(attend(rows=-1), "rows")
    refused(attend(qp=None), "q and out")
    refused(attend(op=None), "q and out")
    refused(attend(ldq=255), "ldq")
    refused(attend(ldo=255), "ldq")
    refused(attend(qp=q.data_ptr() + 1), "aligned")
    refused(attend(heads=3), "heads")
    refused(attend(heads=0), "heads")
    refused(attend(heads=2048), "heads")
    refused(attend(scale=math.inf), "scale")
    refused(attend(scale=math.nan), "scale")
    refused(attend(sinks=-1), "sinks")
    refused(attend(s=B.Sequences(4)), "without table")
    refused(lib.as_attend(ctx._h, None, seqs._ref, 4, q.data_ptr(), 256, 4, 1.0, 0, 0, out.data_ptr(), 256), "cache")
    refused(lib.as_attend(ctx._h, cache._ref, None, 4, q.data_ptr(), 256, 4, 1.0, 0, 0, out.data_ptr(), 256), "sequences")
    refused(prompts(tokens=65), "tokens")
    refused(prompts(tokens=-1), "tokens")
    refused(prompts(at=None), "offsets")
    refused(prompts(at=offsets.data_ptr() + 4), "offsets")
    refused(add(kp=None), "k and v")
    refused(add(ldk=127), "ldk")
    refused(add(tokens=5), "a token a row")
    refused(add(tokens=65, at=offsets.data_ptr()), "tokens")
    refused(add(kp=q.data_ptr() + 1), "aligned")
    refused(add(s=B.Sequences(4)), "table")
    shared = setup(prompts=True)[3]
    refused(prompts(s=shared), "prompt_table", code=UNSUPPORTED)
    for name, value, word in (("k", None, "k and v"), ("v", None, "k and v"), ("k", cache._c.k + 8, "16 bytes"), ("pages", 0, "pages"), ("pages", 1 << 31, "pages"),
                              ("page_size", 0, "page_size"), ("page_size", 24, "page_size"), ("page_size", 1 << 21, "page_size"), ("head_dim", 0, "head_dim"),
                              ("head_dim", 60, "head_dim"), ("head_dim", 264, "head_dim"), ("kv_heads", 0, "kv_heads"), ("kv_heads", 2000, "kv_heads"),
                              ("page_ld", 2047, "page_ld"), ("page_ld", 2052, "16 bytes"), ("page_ld", 1 << 31, "page_ld"), ("dtype", 2, "dtype")):
        c = B.Cache(b.k, b.v)
        setattr(c._c, name, value)
        refused(attend(c=c), word)
    for name, value, word in (("lens", None, "lens"), ("table_ld", 0, "table_ld"), ("table_ld", (1 << 26) + 1, "2^30"), ("lens", b.lens.data_ptr() + 2, "aligned"),
                              ("table", b.table.data_ptr() + 1, "aligned")):
        s = B.Sequences(4, b.table, b.lens)
        setattr(s._c, name, value)
        refused(attend(s=s), word)
    p = setup(prompts=True)
    for name, value, word in (("prompt_lens", None, "prompt_lens"), ("prompt_table_ld", 0, "prompt_table"), ("rows_per_prompt", 0, "rows_per_prompt")):
        s = B.Sequences(4, p[0].table, p[0].lens, p[0].prompt_table, p[0].prompt_lens, 2)
        setattr(s._c, name, value)
        refused(attend(s=s), word)
    torch.cuda.synchronize()
    assert attend() == 0
    torch.cuda.synchronize()
    check(out, q, b)


def test_the_workspace_is_refused_and_then_had():
    b = Batch([3000, 2000], 64, 2, 16, "bf16", seed=2)
    ctx = B.Ctx(2, 100)
    q = torch.randn(2, 256, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    cache, seqs = B.Cache(b.k, b.v), B.Sequences(2, b.table, b.lens)
    # 2 rows of 4 heads, 12 parts of 64 sums and two more words each: 25 KB and less than a MiB, which is what the knob counts in; a
    # batch of 4096 rows is not
    many = Batch([5] * 64, 64, 2, 16, "bf16", prompts=[600], per=64)
    big = B.Ctx(64, 100)
    big.set_tuning("workspace_mib", 1)
    wide = torch.randn(64, 128 * 64, device="cuda").bfloat16()
    with pytest.raises(B.ArithSamplingError, match="workspace") as e:
        B.as_attend(big, B.Cache(many.k, many.v), B.Sequences(64, many.table, many.lens, many.prompt_table, many.prompt_lens, 64), wide, torch.empty_like(wide))
    assert e.value.code == ALLOC
    big.set_tuning("workspace_mib", 0)
    got = torch.empty_like(wide)
    B.as_attend(big, B.Cache(many.k, many.v), B.Sequences(64, many.table, many.lens, many.prompt_table, many.prompt_lens, 64), wide, got)
    check(got, wide, many, rows=[0, 63])
    B.as_attend(ctx, cache, seqs, q, out)
    check(out, q, b)


def capture(stream, work):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        work()
    return graph


@pytest.mark.parametrize("kind", ["attend", "shared", "prompts"])
def test_captured_calls_replay_with_new_lengths_and_contents(kind):
    """Parts and their joining under capture, replayed between eager calls of the same and of smaller sizes."""
    side = torch.cuda.Stream()
    b = Batch([4000, 2500, 3100, 77], 64, 2, 16, "bf16", prompts=[700, 90] if kind == "shared" else None, per=2, seed=5)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx = B.Ctx(64, 100)
        cache = B.Cache(b.k, b.v)
        seqs = B.Sequences(4, b.table, b.lens, b.prompt_table, b.prompt_lens, 2)
        new = [3, 1, 9, 20] if kind == "prompts" else [1] * 4
        offsets = torch.tensor([0] + new, device="cuda").cumsum(0)
        q = torch.randn(sum(new), 512, device="cuda").bfloat16()
        kv = torch.randn(sum(new), 256, device="cuda").bfloat16()
        out = torch.zeros_like(q)

        def work():
            if kind == "prompts":
                B.as_cache_add(ctx, cache, seqs, kv[:, :128], kv[:, 128:], offsets)
                B.as_attend_prompts(ctx, cache, seqs, q, offsets, out)
            else:
                B.as_cache_add(ctx, cache, seqs, kv[:, :128], kv[:, 128:])
                B.as_attend(ctx, cache, seqs, q, out)

        work()
        side.synchronize()
        graph = capture(side, work)
        small = Batch([300], 64, 1, 16, "bf16", seed=6)
        q_small = torch.randn(1, 64, device="cuda").bfloat16()
        out_small = torch.zeros_like(q_small)
        for lens in ([4000, 2500, 3100, 77], [1000, 20, 3000, 30], [3999, 60, 9, 76]):
            q.normal_()
            kv.normal_()
            b.lens.copy_(torch.tensor(lens, dtype=torch.int32))
            b.own = lens
            out.zero_()
            graph.replay()
            side.synchronize()
            got = out.clone()
            check(got, q, b, offsets=offsets.tolist())
            work()
            side.synchronize()
            assert torch.equal(got, out)
            B.as_attend(ctx, B.Cache(small.k, small.v), B.Sequences(1, small.table, small.lens), q_small, out_small)
            check(out_small, q_small, small)
    torch.cuda.synchronize()


def test_two_contexts_on_two_streams():
    """Their calls overlap, each on a workspace and tensors of its own."""
    batches = [Batch([6000, 5000, 10], 128, 2, 16, "bf16", seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    made = []
    for b, stream in zip(batches, streams):
        with torch.cuda.stream(stream):
            q = torch.randn(3, 1024, device="cuda").bfloat16()
            made.append((B.Ctx(3, 100, stream=stream), B.Cache(b.k, b.v), B.Sequences(3, b.table, b.lens), q, [torch.zeros_like(q) for _ in range(20)]))
    for i in range(20):
        for (ctx, cache, seqs, q, out), stream in zip(made, streams):
            with torch.cuda.stream(stream):
                B.as_attend(ctx, cache, seqs, q, out[i])
    torch.cuda.synchronize()
    for b, (_, _, _, q, out) in zip(batches, made):
        check(out[0], q, b)
        assert all(torch.equal(o, out[0]) for o in out)


@pytest.mark.parametrize("form", ["bf16", "bf16 16", "f32"])
def test_far_pages(form):
    """A cache of more than 2^32 values, the tokens in its last pages; rows of q and out more than 2^31 values apart from the first."""
    dim, kv, page = 128, 1, 16
    dtype = torch.float32 if form == "f32" else torch.bfloat16
    pages = (1 << 32) // (kv * page * dim) + 64
    k, v = (torch.zeros(pages, kv, page, dim, dtype=dtype, device="cuda") for _ in range(2))
    own, prompts = [70, 33], [100]
    b = Batch(own, dim, kv, page, form, prompts=prompts, per=2, seed=1)
    shift = pages - b.k.shape[0]
    k[shift:], v[shift:] = b.k, b.v
    table, prompt_table = b.table + shift, b.prompt_table + shift          # (entries past a length are looked at by nobody)
    far = (1 << 31) + 4096
    wide = torch.empty(far + 4096, dtype=dtype, device="cuda")
    q = wide.as_strided((2, 2048), (far, 1))
    out = q[:, 1024:]
    q[:, :1024].normal_()
    ctx = B.Ctx(256, 100)
    if b.shape:
        ctx.set_tuning("attend_shape", b.shape)
    cache = B.Cache(k, v)
    new = torch.randn(2, 256, device="cuda").to(dtype)
    seqs = B.Sequences(2, table, b.lens, prompt_table, b.prompt_lens, 2)
    B.as_cache_add(ctx, cache, seqs, new[:, :128], new[:, 128:])
    for r in range(2):
        p, i = b.place(r, prompts[0] + own[r] - 1)
        b.k[p, 0, i], b.v[p, 0, i] = new[r, :128], new[r, 128:]
    assert torch.equal(k[shift:].nan_to_num(nan=9.0), b.k.nan_to_num(nan=9.0)) and not bool(k[:1000].any())
    B.as_attend(ctx, cache, seqs, q[:, :1024], out)
    check(out, q[:, :1024], b)
    # and as prompts
    n = 33
    alone = Batch([n], dim, kv, page, form, seed=2)
    shift = pages - alone.k.shape[0]
    k[shift:], v[shift:] = alone.k, alone.v
    x = torch.randn(n, 1024, device="cuda").to(dtype)
    y = torch.zeros_like(x)
    B.as_attend_prompts(ctx, cache, B.Sequences(1, alone.table + shift, alone.lens), x, torch.tensor([0, n], device="cuda"), y)
    check(y, x, alone, offsets=[0, n])


@pytest.mark.parametrize("form", ["bf16", "bf16 16", "bf16 128", "f32"])
def test_queries_that_start_anywhere(form):
    b = Batch([100, 3, 40], 64, 2, 16, form, prompts=[50], per=3, seed=4)
    ctx = B.Ctx(3, 100)
    if b.shape:
        ctx.set_tuning("attend_shape", b.shape)
    q = torch.randn(3 * 257 + 8, device="cuda").to(b.dtype)[3:3 + 3 * 257].view(3, 257)[:, :256]
    out = torch.full((3 * 259 + 8,), 7.0, device="cuda", dtype=b.dtype)
    to = out[1:1 + 3 * 259].view(3, 259)[:, :256]
    B.as_attend(ctx, B.Cache(b.k, b.v), B.Sequences(3, b.table, b.lens, b.prompt_table, b.prompt_lens, 3), q, to)
    check(to, q, b)
    assert bool((out[1:1 + 3 * 259].view(3, 259)[:, 256:] == 7).all()) and float(out[0]) == 7.0


def test_tables_wider_than_their_lengths():
    """Room for far more than there is: the keys that are there are split all the same, and parts with nothing say so."""
    b = Batch([5000, 1, 0, 300], 64, 1, 16, "bf16", room=1 << 16)
    ctx = B.Ctx(64, 100)
    q = torch.randn(4, 128, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    B.as_attend(ctx, B.Cache(b.k, b.v), B.Sequences(4, b.table, b.lens), q, out)
    check(out, q, b)
    offsets = torch.tensor([0, 1, 2, 2, 4], device="cuda")
    out.fill_(7.0)
    B.as_attend_prompts(ctx, B.Cache(b.k, b.v), B.Sequences(4, b.table, b.lens), q, offsets, out)
    check(out, q, b, offsets=offsets.tolist())
