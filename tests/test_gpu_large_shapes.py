"""Logits and products of the sizes that a batch has, whose kernels take other forms than small ones do: shaped rows by waves of
1024 columns, through the caches and past them, with few and with most columns seen; and products whose blocks take two or three
256 x 256 tiles each, one's loads under the other's epilogue, whole tiles before partial ones and the reverse.

The references are the definitions in 64 bits, on the GPU; tolerances as derived in test_gpu_linear and test_gpu_shaping."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import apart, problem
from test_gpu_shaping import ALL, SETS, inputs, to_shaping

pytestmark = pytest.mark.gpu

INF = float("inf")


def many_seen(p, rng, upto):
    """Most of the first `upto` columns seen and counted, as in a vocabulary ordered by frequency."""
    here = rng.random((p["counts"].shape[0], upto)) < 0.8
    p["counts"][:, :upto] = np.where(here, rng.integers(0, 4, here.shape), 0)
    p["seen"][:, :upto] = here
    return p


def shaped64(y, p, names):
    """[rows, n] in float64 shaped, and the magnitudes that its roundings go by."""
    t = {k: torch.from_numpy(p[k]).cuda() for k in names if k not in ("seen", "mask")}
    size = y.abs()
    if "repetition" in names:
        th = t["repetition"].double()[:, None]
        y = torch.where(torch.from_numpy(p["seen"]).cuda(), torch.where(y > 0, y / th, y * th), y)
        size = torch.maximum(size, y.abs())
    if "frequency" in names:
        d = t["counts"].double() * t["frequency"].double()[:, None]
        y, size = y - d, size + d.abs()
    if "presence" in names:
        d = (t["counts"] > 0).double() * t["presence"].double()[:, None]
        y, size = y - d, size + d.abs()
    rows = torch.arange(y.shape[0], device="cuda")
    if "bias" in names:
        ids = t["bias_ids"].long().clamp_max(2) if "bias_ids" in names else rows
        d = torch.where((ids >= 0)[:, None], t["bias"].double()[ids.clamp_min(0)], 0.0)
        y, size = y + d, size + d.abs()
    if "mask" in names:
        ids = t["mask_ids"].long().clamp_max(3) if "mask_ids" in names else rows
        free = torch.from_numpy(p["mask"]).cuda()[ids.clamp_min(0)] | (ids < 0)[:, None]
        y = y.masked_fill(~free, -INF)
    return y, size


def compare(out, want, size, extra, what):
    tol = 6 * 2.0 ** -24 * size + extra
    if out.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    got, fine = out.double(), torch.isfinite(want)
    bad = torch.where(fine, ~((got - want).abs() <= tol), got != want)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} off, first at {bad.nonzero()[:3].tolist()}"


def finished_rows(rows, seed):
    return (torch.rand(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) < 0.2).to(torch.uint8)


# pad: rows a million elements apart are a tensor that no cache holds, which is read and written past them
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1), (1000001, 5)])
@pytest.mark.parametrize("names", SETS, ids=lambda s: "+".join(s) or "none")
@pytest.mark.parametrize("few", [True, False])
def test_shape_by_waves_of_1024_columns(dtype, pad, shift, names, few):
    rows, V = 70, 33333
    rng = np.random.default_rng(pad + few)
    p = inputs(rows, V, seed=pad)
    if names in (("bias",), ("mask",)):      # no ids: a row each
        p["bias"], p["mask"] = p["bias"][np.arange(rows) % 3], p["mask"][np.arange(rows) % 4]
    if not few:
        many_seen(p, rng, 20000)
    x = (torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(pad)) * 3).to(dtype)
    flat = torch.full((rows * (V + pad) + shift + 16,), 77.0, dtype=dtype, device="cuda")
    wide = flat[shift:shift + rows * (V + pad)].view(rows, V + pad)
    fin = finished_rows(rows, pad)
    B.as_shape_logits(B.Ctx(rows, V, dtype), apart(x, pad, shift), to_shaping(p, rows, V, names, finished=fin), wide[:, :V])
    want, size = shaped64(x.double(), p, names)
    live = fin == 0
    compare(wide[:, :V][live], want[live], size[live], 0.0, (pad, names))
    untouched = live[:, None] & (want == x.double())
    assert torch.equal(wide[:, :V][untouched], x[untouched])
    wide[live, :V] = 77.0
    assert bool((flat == 77.0).all()), "wrote outside its columns, or a finished row"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [2056, 33333])
def test_shape_in_place_with_most_columns_seen(dtype, V):
    rows = 70
    p = many_seen(inputs(rows, V, seed=V), np.random.default_rng(V), V * 2 // 3)
    x = (torch.randn(rows, V, device="cuda") * 3).to(dtype)
    y = x.clone()
    B.as_shape_logits(B.Ctx(rows, V, dtype), y, to_shaping(p, rows, V, ALL), y)
    want, size = shaped64(x.double(), p, ALL)
    compare(y, want, size, 0.0, V)


# k: two and three stages of 64, the fewest that there are behind a tile's end
SIZES = [(2305, 128, 8200), (4100, 192, 9001), (300, 128, 70001)]


def large(rows, form=6):
    ctx = B.Ctx(rows, 16, torch.float32)
    ctx.set_tuning("linear_shape", form)
    return ctx


def sums64(x, W):
    x, Wt = x.double(), W.double().t().contiguous()
    return x @ Wt, ((x ** 2) @ (Wt ** 2)).sqrt()


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act,with_residual", [("none", False), ("gelu", False), ("none", True), ("gelu", True)])
def test_blocks_of_several_tiles(rows, k, n, out_dtype, act, with_residual):
    x, W, b, r = problem(rows, k, n, torch.bfloat16, out_dtype, seed=rows, residual=True)
    out = torch.full((rows, n + 3), 77.0, dtype=out_dtype, device="cuda")
    B.as_linear(large(rows), B.Layer(W, bias=b, act=act, scale=0.5), x, out[:, :n], residual=r if with_residual else None)
    s, q = sums64(x, W)
    z = 0.5 * s + b.double()
    y = 0.5 * z * torch.special.erfc(-z / 2 ** 0.5) if act == "gelu" else z
    tol = 1.13 * 8 * k ** 0.5 * 2.0 ** -23 * 0.5 * q + 2.0 ** -18 * y.abs() + 2.0 ** -22 * z.abs()
    if with_residual:
        y = y + r.double()
        tol = tol + 2.0 ** -21 * (y.abs() + r.double().abs())
    compare(out[:, :n], y, torch.zeros_like(y), tol, (rows, k, n, act))
    assert bool((out[:, n:] == 77.0).all()), "wrote outside its columns"


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("names", [ALL, ("seen", "repetition", "mask", "mask_ids"), ("seen", "counts", "frequency", "presence")],
                         ids=lambda s: "+".join(s))
@pytest.mark.parametrize("some_finished", [False, True])
def test_blocks_of_several_shaped_tiles(rows, k, n, out_dtype, names, some_finished):
    x, W, b, _ = problem(rows, k, n, torch.bfloat16, out_dtype, seed=rows)
    # few columns seen, and so many of the first that a wave's list does not hold them
    p = many_seen(inputs(rows, n, seed=n), np.random.default_rng(n), 300)
    fin = finished_rows(rows, n) if some_finished else torch.zeros(rows, dtype=torch.uint8, device="cuda")
    out = torch.full((rows, n + 3), 77.0, dtype=out_dtype, device="cuda")
    B.as_linear(large(rows), B.Layer(W, bias=b, act="softcap", act_arg=5.0), x, out[:, :n],
                shaping=to_shaping(p, rows, n, names, finished=fin if some_finished else None))
    s, q = sums64(x, W)
    z = s + b.double()
    extra = 8 * 1.13 * k ** 0.5 * 2.0 ** -23 * q + 2.0 ** -18 * z.abs() + 2.0 ** -22 * z.abs()
    if "repetition" in names:
        th = torch.from_numpy(p["repetition"]).cuda().double()[:, None]
        extra = extra * torch.maximum(th, 1 / th)
    want, size = shaped64(5.0 * torch.tanh(z / 5.0), p, names)
    live = fin == 0
    compare(out[:, :n][live], want[live], size[live], extra[live], (rows, k, n))
    assert bool((out[~live] == 77.0).all()) and bool((out[:, n:] == 77.0).all()), "wrote where nothing is to be"
