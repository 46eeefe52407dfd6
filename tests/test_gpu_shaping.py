"""Shaped logits and token histories against their definitions: as_shape_logits and as_linear with a shaping in 64 bits, the
histories exactly.

Tolerance of a shaped logit, from the arithmetic: at most six fp32 operations, each rounding by 2^-24 of what it handles
(the logit with its penalty, the terms subtracted and added): 6 * 2^-24 of the sum of their magnitudes; and one rounding to
the storage type, 2^-8 of the result in bf16.  What nothing touches keeps its bits."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import binding as B
from test_gpu_linear import act64, apart

pytestmark = pytest.mark.gpu

INF = float("inf")


def pack(bits):
    """bool [rows, n] -> int32 words [rows, ceil(n / 32)] on the GPU."""
    rows, n = bits.shape
    whole = np.zeros((rows, (n + 31) // 32 * 32), dtype=np.uint8)
    whole[:, :n] = bits
    return torch.from_numpy(np.packbits(whole, axis=1, bitorder="little").view(np.int32)).cuda()


def inputs(rows, V, seed, L=20):
    rng = np.random.default_rng(seed)
    counts = np.zeros((rows, V), dtype=np.int32)
    for r in range(rows):
        np.add.at(counts[r], rng.integers(0, V, size=L) * rng.integers(0, 2, size=L), 1)
    seen = counts > 0
    seen[rng.random((rows, V)) < 0.05] = True
    bias = np.where(rng.random((3, V)) < 0.1, rng.normal(0, 4, (3, V)), 0).astype(np.float32)
    bias[rng.random((3, V)) < 0.02] = -INF
    mask = rng.random((4, V)) < np.array([[0.5], [0.95], [0.0], [1.0]])
    f = lambda lo, hi: rng.uniform(lo, hi, rows).astype(np.float32)  # noqa: E731
    return {"seen": seen, "counts": counts, "repetition": f(0.7, 1.6), "presence": f(-0.5, 1), "frequency": f(-0.5, 1),
            "bias": bias, "bias_ids": rng.integers(-2, 3, rows).astype(np.int32),
            "mask": mask, "mask_ids": rng.integers(-2, 4, rows).astype(np.int32)}


def to_shaping(p, rows, V, names, **more):
    t = {}
    for name in names:
        t[name] = pack(p[name]) if name in ("seen", "mask") else torch.from_numpy(p[name]).cuda()
    return B.Shaping(rows, V, **t, **more)


def shaped64(y, p, names):
    """float64 [rows, V] shaped, and the magnitudes that its roundings go by."""
    y = y.copy()
    size = np.abs(y)
    rows = y.shape[0]
    with np.errstate(invalid="ignore"):
        if "repetition" in names:
            th = p["repetition"].astype(np.float64)[:, None]
            y = np.where(p["seen"], np.where(y > 0, y / th, y * th), y)
            size = np.maximum(size, np.abs(y))
        for name, n in (("frequency", p["counts"]), ("presence", (p["counts"] > 0))):
            if name in names:
                d = n * p[name].astype(np.float64)[:, None]
                y, size = y - d, size + np.abs(d)
        for name in ("bias", "mask"):
            if name not in names:
                continue
            ids = p[name + "_ids"] if name + "_ids" in names else np.arange(rows) if p[name].shape[0] > 1 else np.zeros(rows, int)
            ids = np.minimum(ids, p[name].shape[0] - 1)
            rowsof = p[name][np.maximum(ids, 0)]
            if name == "bias":
                d = np.where((ids >= 0)[:, None], rowsof.astype(np.float64), 0.0)
                y, size = y + d, size + np.abs(d)
            else:
                y = np.where(rowsof | (ids < 0)[:, None], y, -INF)
    return y, size


def compare(out, want, size, dtype, what, extra=0.0):
    got = out.double().cpu().numpy()
    ok = np.isnan(got) == np.isnan(want)
    assert ok.all(), f"{what}: NaN at other places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{what}: infinities"
    fine = np.isfinite(want)
    tol = 6 * 2.0 ** -24 * size + extra
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    with np.errstate(invalid="ignore"):
        bad = fine & ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} off, first at {np.argwhere(bad)[:3].tolist()}"


ALL = ("seen", "counts", "repetition", "presence", "frequency", "bias", "bias_ids", "mask", "mask_ids")
SETS = [ALL, ("seen", "repetition"), ("seen", "counts", "presence"), ("seen", "counts", "frequency"), ("bias", "bias_ids"),
        ("mask", "mask_ids"), ("bias",), ("mask",), ()]
WIDTHS = [1, 2, 7, 8, 9, 31, 32, 33, 100, 2047, 2048, 2056, 4101, 9000]


@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("names", SETS, ids=lambda s: "+".join(s) or "none")
def test_shape(V, dtype, names):
    rows = 5
    p = inputs(rows, V, seed=V)
    if names in (("bias",), ("mask",)):      # no ids: a row each
        p["bias"], p["mask"] = p["bias"][[0, 1, 2, 0, 1]], p["mask"][[0, 1, 2, 3, 0]]
    x = (torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)) * 3).to(dtype)
    out = torch.full((rows, V), 77.0, dtype=dtype, device="cuda")
    B.as_shape_logits(B.Ctx(rows, V, dtype), x, to_shaping(p, rows, V, names), out)
    want, size = shaped64(x.double().cpu().numpy(), p, names)
    compare(out, want, size, dtype, (V, names))
    same = torch.from_numpy(want == x.double().cpu().numpy()).cuda()
    assert torch.equal(out[same], x[same])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad_in,shift_in,pad_out,shift_out", [(0, 0, 0, 0), (1, 0, 1, 0), (0, 1, 5, 0), (3, 2, 0, 7), (8, 8, 8, 16)])
@pytest.mark.parametrize("rows,V", [(1, 4101), (6, 333), (40, 2050)])
def test_shape_strides(dtype, pad_in, shift_in, pad_out, shift_out, rows, V):
    p = inputs(rows, V, seed=rows)
    x = (torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)) * 3).to(dtype)
    flat = torch.full((rows * (V + pad_out) + shift_out + 16,), 77.0, dtype=dtype, device="cuda")
    out = flat[shift_out:shift_out + rows * (V + pad_out)].view(rows, V + pad_out)[:, :V]
    B.as_shape_logits(B.Ctx(rows, V, dtype), apart(x, pad_in, shift_in), to_shaping(p, rows, V, ALL), out)
    want, size = shaped64(x.double().cpu().numpy(), p, ALL)
    compare(out, want, size, dtype, (rows, V))
    flat[shift_out:shift_out + rows * (V + pad_out)].view(rows, V + pad_out)[:, :V] = 77.0
    assert bool((flat == 77.0).all()), "wrote outside its columns"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_shape_in_place_finished_and_one_table_row(dtype):
    rows, V = 9, 3001
    p = inputs(rows, V, seed=4)
    p["bias"], p["mask"] = p["bias"][:1], p["mask"][:1]
    names = tuple(n for n in ALL if not n.endswith("_ids"))
    fin = torch.tensor([0, 1, 0, 0, 7, 0, 0, 1, 0], dtype=torch.uint8, device="cuda")
    x = (torch.randn(rows, V, device="cuda") * 3).to(dtype)
    y = x.clone()
    B.as_shape_logits(B.Ctx(rows, V, dtype), y, to_shaping(p, rows, V, names, finished=fin), y)
    done = fin.bool()
    assert torch.equal(y[done], x[done])
    want, size = shaped64(x.double().cpu().numpy(), p, names)
    live = ~done.cpu().numpy()
    compare(y[~done], want[live], size[live], dtype, "in place")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_shape_values_that_are_no_numbers(dtype):
    """Infinities and NaN: forbidden places are -inf whatever was there, the others go by fp32's rules; ids past the
    tables take the last row; a row may be left with nothing, and a step on it stays in range."""
    rows, V = 6, 1000
    p = inputs(rows, V, seed=9)
    p["mask_ids"] = np.array([0, 2, 99, -5, 1, 2], dtype=np.int32)
    p["bias_ids"] = np.array([0, 50, -1, 2, 1, 0], dtype=np.int32)
    lowest = torch.finfo(dtype).min
    x = torch.randn(rows, V, device="cuda").to(dtype)
    x[:, 0:40] = -INF
    x[:, 40:80] = float("nan")
    x[:, 80:100] = INF
    x[:, 100:140] = lowest
    p["bias"][:, 80:100] = 1.0               # (inf - inf is NaN on both sides, but says little)
    out = torch.empty_like(x)
    ctx = B.Ctx(rows, V, dtype)
    B.as_shape_logits(ctx, x, to_shaping(p, rows, V, ALL), out)
    with np.errstate(all="ignore"):
        want, size = shaped64(x.double().cpu().numpy(), p, ALL)
        big = np.abs(want) > float(torch.finfo(dtype).max)               # the lowest value, made larger: past the type
        want[big] = np.sign(want[big]) * INF
        near = (np.abs(want) > 0.98 * -lowest) & np.isfinite(want)       # on the edge either may come
    got = out.double().cpu().numpy()
    want[near] = got[near]
    compare(out, want, np.where(np.isfinite(size), size, 0), dtype, "no numbers")
    assert bool((out[1] == -INF).all()) and bool((out[5] == -INF).all())
    tok = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    codes = torch.full((rows,), 0.5, device="cuda")
    B.as_step(ctx, out, codes, 1.0, 0, 1.0, tok, codes)
    assert bool(((tok >= 0) & (tok < V)).all())


@pytest.mark.parametrize("names", SETS, ids=lambda s: "+".join(s) or "none")
@pytest.mark.parametrize("rows,k,n", [(1, 64, 33), (16, 512, 2000), (70, 128, 4101), (600, 256, 777), (1030, 192, 2600)])
@pytest.mark.parametrize("types", ["bf16", "bf16_f32", "f32"])
def test_linear_shaped(names, rows, k, n, types):
    dtype = torch.float32 if types == "f32" else torch.bfloat16
    out_dtype = torch.bfloat16 if types == "bf16" else torch.float32
    p = inputs(rows, n, seed=n)
    if names in (("bias",), ("mask",)):
        p["bias"], p["mask"] = p["bias"][:1], p["mask"][:1]
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, k, device="cuda", generator=g).to(dtype)
    W = (torch.randn(n, k, device="cuda", generator=g) * (3.0 / k ** 0.5)).to(dtype)
    fin = (torch.rand(rows, device="cuda", generator=g) < 0.2).to(torch.uint8)
    out = torch.full((rows, n), 77.0, dtype=out_dtype, device="cuda")
    B.as_linear(B.Ctx(rows, 16, torch.float32), B.Layer(W, act="softcap", act_arg=5.0), x, out,
                shaping=to_shaping(p, rows, n, names, finished=fin))
    z = x.double().cpu() @ W.double().cpu().t()
    q = ((x.double().cpu() ** 2) @ (W.double().cpu().t() ** 2)).sqrt()
    y = act64(z, "softcap").numpy()
    extra = (1.13 * 8 * k ** 0.5 * 2.0 ** -23 * q + 2.0 ** -18 * z.abs() + 2.0 ** -22 * z.abs()).numpy()      # (as for a layer alone)
    if "repetition" in names:
        extra = extra * np.maximum(p["repetition"], 1 / p["repetition"]).astype(np.float64)[:, None]
        # a sum within its tolerance of zero may be taken for one of the other sign: the penalty of either is within it
    want, size = shaped64(y, p, names)
    live = (fin == 0).cpu().numpy()
    compare(out[fin == 0], want[live], size[live], out_dtype, (names, rows, k, n, types), extra[live])
    assert bool((out[fin != 0] == 77.0).all()), "wrote a finished row"


def history64(rows, V, prompts, offsets, per, tokens, lens):
    counts = np.zeros((rows, V), dtype=np.int32)
    seen = np.zeros((rows, V), dtype=bool)
    for r in range(rows):
        if prompts is not None:
            t = prompts[offsets[r // per]:offsets[r // per + 1]]
            seen[r, t[(t >= 0) & (t < V)]] = True
        if tokens is not None:
            t = tokens[r, :lens[r]]
            np.add.at(counts[r], t[(t >= 0) & (t < V)], 1)
    return seen | (counts > 0), counts


@pytest.mark.parametrize("V", [1, 31, 33, 1000, 8192, 8193, 20000, 70001])
@pytest.mark.parametrize("prompts,per,P,T", [(1, 1, 0, 0), (1, 1, 1, 1), (3, 2, 50, 9), (2, 5, 700, 0), (4, 1, 0, 300), (1, 3, 5000, 3000)])
def test_history_set_and_add(V, prompts, per, P, T):
    rows = prompts * per
    rng = np.random.default_rng(V + P)
    ctx = B.Ctx(rows, V, torch.float32)
    words = (V + 31) // 32
    seen = torch.zeros(rows, words + 1, dtype=torch.int32, device="cuda")[:, :words]
    counts = torch.zeros(rows, V + 3, dtype=torch.int32, device="cuda")[:, :V]
    for turn in range(3):                    # over what the turn before has left
        plens = rng.integers(0, P + 1, prompts)
        offsets = np.concatenate([[0], np.cumsum(plens)]).astype(np.int64)
        # a few tokens are frequent, some lie outside the vocabulary
        pt = np.minimum(rng.integers(-2, V + 3, max(1, offsets[-1])), rng.integers(0, V + 3, max(1, offsets[-1]))).astype(np.int32)
        tt = np.minimum(rng.integers(-2, V + 3, (rows, T)), rng.integers(0, V + 3, (rows, T))).astype(np.int32)
        lens = rng.integers(0, T + 1, rows).astype(np.int32)
        tok_dev = torch.from_numpy(tt).cuda()
        B.as_history_set(ctx, seen, counts, torch.from_numpy(pt).cuda(), torch.from_numpy(offsets).cuda(), per,
                         tok_dev if T else None, torch.from_numpy(lens).cuda() if T else None)
        want_seen, want_counts = history64(rows, V, pt, offsets, per, tt if T else None, lens)
        assert torch.equal(seen, pack(want_seen)) and torch.equal(counts.cpu(), torch.from_numpy(want_counts)), turn
        for _ in range(2):
            last = rng.integers(-1, V + 1, rows).astype(np.int32)
            fin = (rng.random(rows) < 0.3).astype(np.uint8)
            B.as_history_add(ctx, seen, counts, torch.from_numpy(last).cuda(), torch.from_numpy(fin).cuda())
            for r in range(rows):
                if not fin[r] and 0 <= last[r] < V:
                    want_counts[r, last[r]] += 1
                    want_seen[r, last[r]] = True
        assert torch.equal(seen, pack(want_seen)) and torch.equal(counts.cpu(), torch.from_numpy(want_counts)), turn


def test_history_rows_left_alone_no_counts_and_bad_lengths():
    rows, V = 6, 9000
    rng = np.random.default_rng(0)
    ctx = B.Ctx(rows, V, torch.float32)
    seen = torch.zeros(rows, (V + 31) // 32, dtype=torch.int32, device="cuda")
    counts = torch.zeros(rows, V, dtype=torch.int32, device="cuda")
    first = rng.integers(0, V, (rows, 40)).astype(np.int32)
    B.as_history_set(ctx, seen, counts, tokens=torch.from_numpy(first).cuda())
    second = rng.integers(0, V, (rows, 40)).astype(np.int32)
    which = np.array([1, 0, 0, 1, 1, 0], dtype=np.uint8)
    # lengths past the tensor and below zero are brought into it
    lens = np.array([1000, 5, 5, -3, 40, 5], dtype=np.int32)
    B.as_history_set(ctx, seen, counts, tokens=torch.from_numpy(second).cuda(), lens=torch.from_numpy(lens).cuda(),
                     which=torch.from_numpy(which).cuda())
    mixed = np.where(which[:, None] > 0, second, first)
    want_seen, want_counts = history64(rows, V, None, None, 1, mixed, np.where(which > 0, np.clip(lens, 0, 40), 40))
    assert torch.equal(seen, pack(want_seen)) and torch.equal(counts.cpu(), torch.from_numpy(want_counts))
    # offsets outside the prompts too
    prompts = torch.arange(10, dtype=torch.int32, device="cuda")
    bad = torch.tensor([-5, 3, 2, 900], dtype=torch.int64, device="cuda")
    only = torch.zeros_like(seen)
    B.as_history_set(ctx, only, None, prompts, bad, 2)
    want = np.zeros((rows, V), dtype=bool)
    want[0:2, 0:3] = True
    want[4:6, 2:10] = True
    assert torch.equal(only, pack(want))
    B.as_history_add(ctx, only, None, torch.full((rows,), 77, dtype=torch.int32, device="cuda"))
    want[:, 77] = True
    assert torch.equal(only, pack(want))


def test_shaped_decode_under_a_graph():
    """History, layer with shaping, step: captured once, replayed, against the same calls made one by one."""
    rows, k, V, steps = 8, 128, 3001, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    W = (torch.randn(V, k, device="cuda", generator=g) * 0.2).to(torch.bfloat16)
    emb = torch.randn(V, k, device="cuda", generator=g).to(torch.bfloat16)
    layer = B.Layer(W)
    start = torch.rand(rows, device="cuda", generator=g)

    def state():
        s = {"seen": torch.zeros(rows, (V + 31) // 32, dtype=torch.int32, device="cuda"),
             "counts": torch.zeros(rows, V, dtype=torch.int32, device="cuda"),
             "tok": torch.arange(rows, dtype=torch.int32, device="cuda"), "codes": start.clone(),
             "logits": torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")}
        s["shaping"] = B.Shaping(rows, V, seen=s["seen"], counts=s["counts"], repetition=torch.full((rows,), 1.3, device="cuda"),
                                 frequency=torch.full((rows,), 0.4, device="cuda"))
        return s

    def step(ctx, s):
        B.as_history_add(ctx, s["seen"], s["counts"], s["tok"])
        B.as_linear(ctx, layer, emb[s["tok"].long()], s["logits"], shaping=s["shaping"])
        B.as_step(ctx, s["logits"], s["codes"], 0.9, 0, 1.0, s["tok"], s["codes"])

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx = B.Ctx(rows, V, torch.bfloat16, stream=side)
        one, two = state(), state()
        want = []
        for _ in range(steps):
            step(ctx, one)
            want.append((one["tok"].clone(), one["codes"].clone(), one["counts"].clone()))
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(ctx, two)
        for t in range(steps):
            graph.replay()
            side.synchronize()
            for a, b in zip(want[t], (two["tok"], two["codes"], two["counts"])):
                assert torch.equal(a, b), t
            (torch.randn(64, 64, device="cuda") @ torch.randn(64, 64, device="cuda")).sum()
    torch.cuda.synchronize()


def test_refusals():
    rows, V = 4, 100
    p = inputs(rows, V, seed=1)
    ctx = B.Ctx(rows, V, torch.float32)
    x = torch.zeros(rows, V, device="cuda")
    out = torch.full((rows, V), 7.0, device="cuda")
    for names in (("repetition",), ("presence",), ("seen", "frequency")):
        with pytest.raises(B.ArithSamplingError, match="need"):
            B.as_shape_logits(ctx, x, to_shaping(p, rows, V, names), out)
    for name in ("bias", "mask"):            # three rows of a table for four rows
        with pytest.raises(B.ArithSamplingError, match="_rows"):
            B.as_shape_logits(ctx, x, B.Shaping(rows, V, **{name: pack(p[name][:3]) if name == "mask" else torch.from_numpy(p[name]).cuda()}), out)
    with pytest.raises(ValueError):
        B.Shaping(rows, V, seen=torch.zeros(rows, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        B.Shaping(rows, V, counts=torch.zeros(rows, 99, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        B.Shaping(rows, V, repetition=torch.ones(3, device="cuda"))
    with pytest.raises(TypeError):
        B.Shaping(rows, V, repetition=torch.ones(4, device="cuda", dtype=torch.float64))
    shaping = B.Shaping(rows, V)
    with pytest.raises(TypeError):
        B.as_shape_logits(ctx, x.bfloat16(), shaping, out)
    with pytest.raises(ValueError):
        B.as_shape_logits(ctx, x, shaping, out[:, :99])
    with pytest.raises(ValueError):
        B.as_shape_logits(ctx, x, B.Shaping(3, V), out)
    with pytest.raises(B.ArithSamplingError, match="max_rows"):
        B.as_shape_logits(B.Ctx(3, V, torch.float32), x, shaping, out)
    seen = torch.zeros(rows, 4, dtype=torch.int32, device="cuda")
    counts = torch.zeros(rows, V, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        B.as_history_set(ctx, seen[:, :3], counts)
    with pytest.raises(TypeError):
        B.as_history_set(ctx, seen, counts.long())
    with pytest.raises(ValueError):
        B.as_history_set(ctx, seen, counts, torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), 1)
    with pytest.raises(B.ArithSamplingError, match="rows_per_prompt"):
        B.as_history_set(ctx, seen, counts, torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int64, device="cuda"), -1)
    with pytest.raises(ValueError):
        B.as_history_add(ctx, seen, counts, torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(B.ArithSamplingError, match="max_rows"):
        B.as_history_add(B.Ctx(3, V, torch.float32), seen, counts, torch.zeros(rows, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and not bool(counts.any()) and not bool(seen.any())
