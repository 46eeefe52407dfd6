"""as_linear against the layer's formula in 64 bits, at the sizes, strides, types and masks where it can go wrong.

Tolerance of one output, from the arithmetic.  The sum of k products is held in fp32: each of its k additions rounds by at
most 2^-23 (a matrix instruction may truncate) of a partial sum, which over independent terms stays within a few times
their root sum square q = sqrt(sum (x w)^2); the roundings are independent, so 8 sqrt(k) 2^-23 q bounds the sum, times the
largest slope of an activation, 1.13.  The activations add 2^-18 of their value (an exponential of an argument rounded to
fp32: up to 40 ulps where the value matters) and 2^-22 of their argument (a published fit of erf, 1.5e-7).  What follows
rounds a few times in fp32 (2^-21 of each term), and the storage type once (2^-8 of the result in bf16)."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu

CAP = 5.0
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu", "softcap"]


def act64(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / 2 ** 0.5)
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "softcap":
        return CAP * torch.tanh(z / CAP)
    return z


def apart(t, pad, shift=0):
    """The same rows `pad` elements further apart, the first `shift` elements into its memory; NaN in between."""
    if not pad and not shift:
        return t
    flat = torch.full((t.shape[0] * (t.shape[1] + pad) + shift + 8,), float("nan"), dtype=t.dtype, device=t.device)
    wide = flat[shift:shift + t.shape[0] * (t.shape[1] + pad)].view(t.shape[0], t.shape[1] + pad)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def check(out, x, W, bias, act, scale, residual, what):
    x, W = x.double(), W.double()
    k = x.shape[1]
    s = scale * (x.cpu() @ W.cpu().t())
    q = abs(scale) * ((x.cpu() ** 2) @ (W.cpu().t() ** 2)).sqrt()
    z = s if bias is None else s + bias.double().cpu()
    y = act64(z, act)
    tol = 1.13 * 8 * k ** 0.5 * 2.0 ** -23 * q + 2.0 ** -18 * y.abs() + 2.0 ** -22 * z.abs()
    if residual is not None:
        r = residual.double().cpu()
        y, tol = y + r, tol + 2.0 ** -21 * (y.abs() + r.abs())
    if out.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (y.abs() + tol)
    far = ((out.double().cpu() - y).abs() - tol).max().item()
    worst = ((out.double().cpu() - y).abs() / (tol + 1e-300)).max().item()
    assert far <= 0, f"{what}: {worst:.2f} of the tolerance"
    assert torch.isfinite(out).all(), what


def problem(rows, k, n, dtype, out_dtype, seed, bias=True, residual=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, k, device="cuda", generator=g).to(dtype)
    W = (torch.randn(n, k, device="cuda", generator=g) * (2.0 / k ** 0.5)).to(dtype)
    b = (torch.randn(n, device="cuda", generator=g) * 0.5).to(dtype) if bias else None
    r = torch.randn(rows, n, device="cuda", generator=g).to(out_dtype) if residual else None
    return x, W, b, r


# rows and columns on either side of every tile of the kernels, k of less than a step, of a step, between steps
SIZES = [(1, 64, 64), (1, 1, 1), (1, 512, 2048), (2, 63, 65), (3, 65, 1), (7, 130, 300), (15, 192, 31), (16, 256, 33),
         (17, 64, 1000), (31, 1000, 129), (33, 128, 255), (64, 2048, 512), (65, 320, 257), (127, 96, 130), (128, 448, 640),
         (129, 64, 96), (200, 520, 1031), (255, 576, 511), (256, 128, 256), (257, 192, 513), (300, 1024, 40),
         (1000, 72, 260), (1024, 512, 2048), (1025, 640, 770)]


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("types", ["bf16", "bf16_f32", "f32"])
def test_sizes(rows, k, n, types):
    dtype = torch.float32 if types == "f32" else torch.bfloat16
    out_dtype = torch.bfloat16 if types == "bf16" else torch.float32
    x, W, b, r = problem(rows, k, n, dtype, out_dtype, seed=rows * 7 + k, residual=True)
    ctx = B.Ctx(rows, 16, torch.float32)
    layer = B.Layer(W, bias=b, act="silu", scale=0.75)
    out = torch.full((rows, n), float("nan"), dtype=out_dtype, device="cuda")
    B.as_linear(ctx, layer, x, out, residual=r)
    check(out, x, W, b, "silu", 0.75, r, (rows, k, n, types))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,k,n", [(5, 128, 200), (300, 256, 520), (2048, 256, 2304)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_activations(act, rows, k, n, dtype):
    x, W, b, _ = problem(rows, k, n, dtype, dtype, seed=len(act) + rows)
    W = W * 2                                # arguments well into the tails
    ctx = B.Ctx(rows, 16, torch.float32)
    out = torch.empty(rows, n, dtype=dtype, device="cuda")
    B.as_linear(ctx, B.Layer(W, bias=b, act=act, act_arg=CAP), x, out)
    check(out, x, W, b, act, 1.0, None, (act, rows, k, n, dtype))


@pytest.mark.parametrize("act,at_minus,at_plus", [("relu", 0.0, 60000.0), ("gelu", 0.0, 60000.0), ("gelu_tanh", 0.0, 60000.0),
                                                  ("silu", 0.0, 60000.0), ("softcap", -CAP, CAP)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_activations_far_out(act, at_minus, at_plus, dtype):
    """Arguments whose exponentials leave fp32: the activations take their limits, no NaN."""
    x = torch.tensor([[-1.0], [1.0]], device="cuda", dtype=dtype)
    W = torch.full((40, 1), 60000.0, device="cuda", dtype=dtype)
    out = torch.empty(2, 40, dtype=dtype, device="cuda")
    B.as_linear(B.Ctx(2, 16, torch.float32), B.Layer(W, act=act, act_arg=CAP), x, out)
    want = torch.tensor([[at_minus], [at_plus]]).to(dtype).float().expand(2, 40)
    assert torch.equal(out.float().cpu(), want), out[:, :2]


@pytest.mark.parametrize("types", ["bf16", "bf16_f32", "f32"])
@pytest.mark.parametrize("rows,k,n", [(1, 320, 77), (9, 128, 1000), (140, 192, 600), (600, 256, 1030)])
@pytest.mark.parametrize("xpad,xshift,wpad,opad,oshift", [(1, 0, 0, 3, 0), (8, 8, 8, 8, 8), (0, 1, 0, 0, 1), (5, 3, 7, 1, 5), (64, 0, 3, 2, 0)])
def test_strides_and_alignment(types, rows, k, n, xpad, xshift, wpad, opad, oshift):
    """Rows that start anywhere; what lies between them is NaN and stays what it was."""
    dtype = torch.float32 if types == "f32" else torch.bfloat16
    out_dtype = torch.bfloat16 if types == "bf16" else torch.float32
    x, W, b, r = problem(rows, k, n, dtype, out_dtype, seed=xpad + n, residual=True)
    flat = torch.full((rows * (n + opad) + oshift + 16,), 77.0, dtype=out_dtype, device="cuda")
    out = flat[oshift:oshift + rows * (n + opad)].view(rows, n + opad)[:, :n]
    B.as_linear(B.Ctx(rows, 16, torch.float32), B.Layer(apart(W, wpad, wpad), bias=b, act="gelu_tanh"), apart(x, xpad, xshift), out,
                residual=apart(r, opad + 1, 1))
    check(out, x, W, b, "gelu_tanh", 1.0, r, (types, rows, k, n))
    wide = flat.clone()
    wide[oshift:oshift + rows * (n + opad)].view(rows, n + opad)[:, :n] = 77.0
    assert bool((wide == 77.0).all()), "wrote outside its columns"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k,n", [(6, 512, 100), (700, 512, 768)])
def test_residual_in_place(dtype, rows, k, n):
    x, W, b, r = problem(rows, k, n, dtype, dtype, seed=3, residual=True)
    out = r.clone()
    B.as_linear(B.Ctx(rows, 16, torch.float32), B.Layer(W, bias=b), x, out, residual=out)
    check(out, x, W, b, "none", 1.0, r, (dtype, rows))


@pytest.mark.parametrize("rows,k,n", [(1, 4096, 64), (4, 8192, 33), (48, 4096, 200), (16384, 64, 40), (40000, 128, 70),
                                      (2, 64, 131100), (520, 128, 20000)])
def test_long_sides(rows, k, n):
    """One side much longer than the others: a long sum, many rows, many columns."""
    x, W, b, _ = problem(rows, k, n, torch.bfloat16, torch.bfloat16, seed=5)
    out = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    B.as_linear(B.Ctx(rows, 16, torch.float32), B.Layer(W, bias=b), x, out)
    check(out, x, W, b, "none", 1.0, None, (rows, k, n))


@pytest.mark.parametrize("types", ["bf16", "f32"])
@pytest.mark.parametrize("rows,k,n", [(3, 256, 300), (40, 1024, 256), (512, 512, 4096), (2049, 256, 8200)])
def test_the_same_bits_again_and_in_any_batch(types, rows, k, n):
    """Calls repeat bit for bit, and NaN or infinite rows of x leave the others as they are."""
    dtype = torch.float32 if types == "f32" else torch.bfloat16
    x, W, b, _ = problem(rows, k, n, dtype, dtype, seed=11)
    ctx, layer = B.Ctx(rows, 16, torch.float32), B.Layer(W, bias=b, act="silu")
    outs = [torch.full((rows, n), float("nan"), dtype=dtype, device="cuda") for _ in range(3)]
    for o in outs:
        B.as_linear(ctx, layer, x, o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    x2 = x.clone()
    x2[1] = float("nan")
    x2[rows - 1] = float("inf")
    B.as_linear(ctx, layer, x2, outs[1])
    keep = [i for i in range(rows) if i not in (1, rows - 1)]
    assert torch.equal(outs[1][keep], outs[0][keep])
    assert bool(torch.isnan(outs[1][1]).all())


def test_nothing_to_do_and_no_bias():
    x, W, _, _ = problem(4, 96, 50, torch.bfloat16, torch.float32, seed=2)
    ctx, layer = B.Ctx(8, 16, torch.float32), B.Layer(W)
    out = torch.full((4, 50), 7.0, device="cuda")
    B.as_linear(ctx, layer, x[:0], out[:0])
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    B.as_linear(ctx, layer, x, out)
    check(out, x, W, None, "none", 1.0, None, "no bias")


def test_other_streams_and_graphs():
    """Work goes to the context's stream; a captured call replays, between eager ones, with what its inputs hold then."""
    rows, k, n = 24, 1000, 300               # rows of x that have to be laid out
    x, W, b, r = problem(rows, k, n, torch.bfloat16, torch.bfloat16, seed=8, residual=True)
    side = torch.cuda.Stream()
    layer = B.Layer(W, bias=b, act="gelu")
    out = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx = B.Ctx(rows, 16, torch.float32, stream=side)
        B.as_linear(ctx, layer, x, out, residual=r)
        side.synchronize()
        check(out, x, W, b, "gelu", 1.0, r, "side stream")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.as_linear(ctx, layer, x, out, residual=r)
        for i in range(4):
            x.copy_(torch.randn(rows, k, device="cuda").to(torch.bfloat16))
            eager = torch.empty_like(out)
            B.as_linear(ctx, layer, x, eager, residual=r)
            out.fill_(float("nan"))
            graph.replay()
            side.synchronize()
            assert torch.equal(out, eager), f"replay {i}"
    torch.cuda.synchronize()


def test_refusals():
    x, W, b, _ = problem(4, 64, 48, torch.bfloat16, torch.bfloat16, seed=1)
    ctx, layer = B.Ctx(4, 16, torch.float32), B.Layer(W, bias=b)
    out = torch.full((4, 48), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        B.as_linear(ctx, layer, x.float(), out)
    with pytest.raises(TypeError):
        B.as_linear(ctx, layer, x, out.half())
    with pytest.raises(TypeError):
        B.as_linear(ctx, layer, x.cpu(), out)
    with pytest.raises(ValueError):
        B.as_linear(ctx, layer, x[:, :63], out)
    with pytest.raises(ValueError):
        B.as_linear(ctx, layer, x, out[:, :47])
    with pytest.raises(ValueError):
        B.as_linear(ctx, layer, x, out[:3])
    with pytest.raises(ValueError):
        B.as_linear(ctx, layer, x.t().contiguous().t(), out)
    with pytest.raises(ValueError):
        B.as_linear(ctx, layer, x[:1].expand(4, 64), out)
    with pytest.raises(TypeError):
        B.as_linear(ctx, layer, x, out, residual=torch.zeros(4, 48, device="cuda"))
    with pytest.raises(B.ArithSamplingError, match="max_rows"):
        B.as_linear(B.Ctx(3, 16, torch.float32), layer, x, out)
    with pytest.raises(B.ArithSamplingError, match="fp32 layer"):
        B.as_linear(ctx, B.Layer(W.float()), x.float(), out)
    with pytest.raises(ValueError, match="activation"):
        B.Layer(W, act="swish")
    with pytest.raises(B.ArithSamplingError, match="cap"):
        B.Layer(W, act="softcap", act_arg=0.0)
    with pytest.raises(B.ArithSamplingError, match="scale"):
        B.Layer(W, scale=float("inf"))
    with pytest.raises(ValueError):
        B.Layer(W, bias=b[:47])
    with pytest.raises(ValueError, match="shaping"):
        B.as_linear(ctx, layer, x, out, shaping=B.Shaping(4, 47))
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()), "a refused call wrote"
