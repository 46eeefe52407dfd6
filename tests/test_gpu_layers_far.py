"""Rows whose offsets pass 32 bits, the profile's count of launches, and calls on a stream that is not their tensors' own."""
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import check, problem

pytestmark = pytest.mark.gpu

FAR = (1 << 31) + 24                         # elements between rows: the third row starts past 2^32


def far(rows, cols, dtype):
    """`rows` rows FAR elements apart, of which only the first columns are ever touched."""
    return torch.empty(rows * FAR, dtype=dtype, device="cuda").view(rows, FAR)[:, :cols]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layer_rows_far_apart(dtype):
    rows, k, n = 3, 192, 300
    x, W, b, _ = problem(rows, k, n, dtype, dtype, seed=1)
    wide_x, wide_out = far(rows, k, dtype), far(rows, n, dtype)
    wide_x.copy_(x)
    B.as_linear(B.Ctx(rows, 16, torch.float32), B.Layer(W, bias=b, act="gelu"), wide_x, wide_out)
    check(wide_out, x, W, b, "gelu", 1.0, None, dtype)


def test_large_tiles_with_outputs_far_apart():
    """Offsets past 32 bits inside a product of the large form: 300 rows of 16 million outputs' distance."""
    rows, k, n = 300, 128, 500
    x, W, b, _ = problem(rows, k, n, torch.bfloat16, torch.bfloat16, seed=2)
    ctx = B.Ctx(rows, 16, torch.float32)
    ctx.set_tuning("linear_shape", 6)
    out = torch.empty(rows * (1 << 24), dtype=torch.bfloat16, device="cuda").view(rows, 1 << 24)[:, :n]
    B.as_linear(ctx, B.Layer(W, bias=b), x, out)
    check(out, x, W, b, "none", 1.0, None, "far outputs")


def test_shaping_and_histories_far_apart():
    rows, V = 3, 5000
    seen, counts = torch.zeros(rows, (V + 31) // 32, dtype=torch.int32, device="cuda"), far(rows, V, torch.int32)
    counts.zero_()
    tokens = torch.randint(0, V, (rows, 50), dtype=torch.int32, device="cuda")
    ctx = B.Ctx(rows, V, torch.bfloat16)
    B.as_history_set(ctx, seen, counts, tokens=tokens)
    B.as_history_add(ctx, seen, counts, tokens[:, 0].contiguous())
    want = torch.zeros(rows, V, dtype=torch.int64, device="cuda").scatter_add_(1, torch.cat([tokens, tokens[:, :1]], 1).long(),
                                                                             torch.ones(rows, 51, dtype=torch.int64, device="cuda"))
    assert torch.equal(counts.long(), want)
    x = far(rows, V, torch.bfloat16)
    x.copy_(torch.randn(rows, V, device="cuda"))
    strength = torch.full((rows,), 0.5, device="cuda")
    B.as_shape_logits(ctx, x.clone(memory_format=torch.contiguous_format), B.Shaping(rows, V, seen=seen, counts=counts, frequency=strength), x)
    near = x.float()
    assert torch.isfinite(near).all()
    plain = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")
    B.as_shape_logits(ctx, x, B.Shaping(rows, V, seen=seen, counts=want.int(), frequency=-strength), plain)
    # there and back again: two roundings to bf16 of numbers of about the same size
    assert (plain.float() - (near + 0.5 * want.float())).abs().max() <= 2.0 ** -8 * (near.abs() + 0.5 * want.float()).max()


def test_profile_counts_a_layer_s_launch():
    x, W, b, _ = problem(20, 128, 300, torch.bfloat16, torch.bfloat16, seed=3)
    ctx, out = B.Ctx(20, 16, torch.float32), torch.empty(20, 300, dtype=torch.bfloat16, device="cuda")
    ctx.profile(True)
    layer = B.Layer(W, bias=b)
    for _ in range(3):
        B.as_linear(ctx, layer, x, out)
    ms, launches, untimed = ctx.profile_read(1)
    assert launches == 3 and untimed == 0 and ms > 0
    check(out, x, W, b, "none", 1.0, None, "profiled")


def test_tensors_of_another_stream():
    """Inputs made on one stream, used on another after an event: the context's stream alone decides where the work goes."""
    x, W, b, _ = problem(64, 256, 512, torch.bfloat16, torch.bfloat16, seed=4)
    torch.cuda.synchronize()
    main, side = torch.cuda.current_stream(), torch.cuda.Stream()
    ctx = B.Ctx(64, 16, torch.float32, stream=side)
    layer, out = B.Layer(W, bias=b, act="silu"), torch.empty(64, 512, dtype=torch.bfloat16, device="cuda")
    for i in range(3):
        y = (x.float() * (i + 1)).to(torch.bfloat16)             # on the main stream
        done = torch.cuda.Event()
        done.record(main)
        side.wait_event(done)
        B.as_linear(ctx, layer, y, out)
        done.record(side)
        main.wait_event(done)
        check(out, y, W, b, "silu", 1.0, None, i)
