"""Every kernel form of as_linear, picked by the tuning knob, at sizes on either side of its tiles, against the formula in 64 bits
(tolerances as derived in test_gpu_linear and test_gpu_shaping)."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import act64, apart, check, problem
from test_gpu_shaping import ALL, compare, inputs, shaped64, to_shaping

pytestmark = pytest.mark.gpu

FORMS = list(range(1, 10))
SIZES = [(1, 64, 33), (5, 192, 130), (16, 512, 300), (33, 1088, 64), (70, 128, 513), (130, 320, 256), (257, 192, 513), (600, 128, 1100),
         (1030, 256, 2600)]


def context(rows, form):
    ctx = B.Ctx(rows, 16, torch.float32)
    ctx.set_tuning("linear_shape", form)
    return ctx


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_plain_and_residual(form, rows, k, n, out_dtype):
    x, W, b, r = problem(rows, k, n, torch.bfloat16, out_dtype, seed=form + n, residual=True)
    ctx, out = context(rows, form), torch.full((rows, n + 3), 77.0, dtype=out_dtype, device="cuda")
    for act, residual in (("none", None), ("gelu", r)):
        B.as_linear(ctx, B.Layer(W, bias=b, act=act, scale=0.5), x, out[:, :n], residual=residual)
        check(out[:, :n], x, W, b, act, 0.5, residual, (form, rows, k, n, act))
        assert bool((out[:, n:] == 77.0).all()), "wrote outside its columns"


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("L", [3, 20, 3000])
def test_shaped(form, rows, k, n, L):
    """Few tokens seen, some, and (nearly) all: the last takes the way for more than a wave's list holds."""
    names = ALL if form % 2 else tuple(x for x in ALL if x not in ("bias", "bias_ids"))
    p = inputs(rows, n, seed=n + L, L=L)
    x, W, b, r = problem(rows, k, n, torch.bfloat16, torch.bfloat16, seed=rows, residual=True)
    for out_dtype, residual in ((torch.bfloat16, None), (torch.float32, None), (torch.bfloat16, r)):
        fin = (torch.rand(rows, device="cuda") < 0.2).to(torch.uint8)
        out = torch.full((rows, n + 5), 77.0, dtype=out_dtype, device="cuda")
        B.as_linear(context(rows, form), B.Layer(W, bias=b, act="softcap", act_arg=5.0), x, out[:, :n], residual=residual,
                    shaping=to_shaping(p, rows, n, names, finished=fin))
        z = x.double().cpu() @ W.double().cpu().t()
        q = ((x.double().cpu() ** 2) @ (W.double().cpu().t() ** 2)).sqrt()
        z = z + b.double().cpu()
        y = act64(z, "softcap")
        extra = (8 * 1.13 * k ** 0.5 * 2.0 ** -23 * q + 2.0 ** -18 * z.abs() + 2.0 ** -22 * z.abs()).numpy()
        if residual is not None:
            y = y + residual.double().cpu()
            extra = extra + (2.0 ** -21 * (y.abs() + residual.double().cpu().abs())).numpy()
        extra = extra * np.maximum(p["repetition"], 1 / p["repetition"]).astype(np.float64)[:, None]
        want, size = shaped64(y.numpy(), p, names)
        live = (fin == 0).cpu().numpy()
        compare(out[:, :n][fin == 0], want[live], size[live], out_dtype, (form, rows, k, n, L), extra[live])
        assert bool((out[fin != 0] == 77.0).all()) and bool((out[:, n:] == 77.0).all()), "wrote where nothing is to be"


@pytest.mark.parametrize("form", FORMS)
def test_rows_of_weights_and_x_apart(form):
    rows, k, n = 150, 256, 420
    x, W, b, _ = problem(rows, k, n, torch.bfloat16, torch.bfloat16, seed=form)
    out = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    for pad, wpad in ((8, 16), (3, 0), (0, 5)):
        B.as_linear(context(rows, form), B.Layer(apart(W, wpad), bias=b), apart(x, pad), out)
        check(out, x, W, b, "none", 1.0, None, (form, pad, wpad))


@pytest.mark.parametrize("form", range(1, 6))
@pytest.mark.parametrize("rows,k,n", [(1, 1, 1), (3, 7, 33), (17, 130, 130), (70, 515, 300), (300, 64, 1031)])
def test_fp32(form, rows, k, n):
    x, W, b, r = problem(rows, k, n, torch.float32, torch.float32, seed=form + n, residual=True)
    p = inputs(rows, n, seed=n, L=20)
    out = torch.full((rows, n + 3), 77.0, device="cuda")
    for xpad, wpad, opad in ((0, 0, 0), (3, 5, 1)):
        B.as_linear(context(rows, form), B.Layer(apart(W, wpad), bias=b, act="silu"), apart(x, xpad), out[:, :n], residual=apart(r, opad))
        check(out[:, :n], x, W, b, "silu", 1.0, r, (form, rows, k, n))
    B.as_linear(context(rows, form), B.Layer(W), x, out[:, :n], shaping=to_shaping(p, rows, n, ALL))
    z = x.double().cpu() @ W.double().cpu().t()
    q = ((x.double().cpu() ** 2) @ (W.double().cpu().t() ** 2)).sqrt()
    extra = (8 * 1.13 * k ** 0.5 * 2.0 ** -23 * q + 2.0 ** -18 * z.abs() + 2.0 ** -22 * z.abs()).numpy()
    extra = extra * np.maximum(p["repetition"], 1 / p["repetition"]).astype(np.float64)[:, None]
    want, size = shaped64(z.numpy(), p, ALL)
    compare(out[:, :n], want, size, torch.float32, (form, rows, k, n), extra)
    assert bool((out[:, n:] == 77.0).all()), "wrote outside its columns"
