"""gelu with fp32 outputs, point by point: sums that are exact (one term, the others zero), so that the activation's own error is
what is left.

Tolerance, from the arithmetic of z h, h = erfc(|z| / sqrt 2) / 2 = t P(t) e^(-z^2 / 2), t = 1 / (1 + p |z| / sqrt 2): t is off by
1.5 * 2^-23 of itself (a reciprocal of 1 ulp, a rounding), which h follows at most 3.05 times; nine terms of P with a sum of
magnitudes of 2.2 times theirs, each rounded once, 10 * 2^-23; the exponential 2^-23 and what its argument is off, 1.25 z^2 2^-24
(two roundings and the constant's); products and the fit itself below 3 * 2^-23 more: 20 * 2^-23 + 1.25 z^2 2^-24 of z h.  Above zero
z (1 - h) has that of its small part and two roundings of its own."""
import pytest
import torch

from paper_2210_15458_amd import binding as B

pytestmark = pytest.mark.gpu


def points(rows, dtype):
    z = torch.cat([torch.linspace(-12, 12, max(2, rows - rows // 3), dtype=torch.float64), torch.linspace(-2, 2, rows // 3, dtype=torch.float64)])[:rows]
    return z.to(dtype).cuda()


@pytest.mark.parametrize("dtype,form,rows", [(torch.float32, f, 4000) for f in range(0, 6)] + [(torch.bfloat16, f, 3000) for f in range(0, 7)] +
                         [(torch.bfloat16, f, 16) for f in (7, 8, 9)])
@pytest.mark.parametrize("residual", [False, True])
def test_gelu(dtype, form, rows, residual):
    k, n = 128, 40
    z = points(rows, dtype)
    x = torch.zeros(rows, k, dtype=dtype, device="cuda")
    x[:, 0] = z
    ctx, out = B.Ctx(rows, 16, torch.float32), torch.empty(rows, n, device="cuda")
    ctx.set_tuning("linear_shape", form)
    B.as_linear(ctx, B.Layer(torch.ones(n, k, dtype=dtype, device="cuda"), act="gelu"), x, out,
                residual=torch.zeros_like(out) if residual else None)
    z = z.double()
    small = (0.5 * z * torch.special.erfc(z.abs() / 2 ** 0.5)).abs()
    y = 0.5 * z * torch.special.erfc(-z / 2 ** 0.5)
    tol = small * (20 * 2.0 ** -23 + 1.25 * z ** 2 * 2.0 ** -24) + torch.where(z > 0, 2.0 ** -23 * y.abs(), 0.0)
    off = (out.double() - y[:, None]).abs().max(dim=1).values
    worst = (off / (tol + 1e-300)).max().item()
    assert bool((off <= tol).all()), f"{worst:.1f} of the tolerance, at {z[(off / (tol + 1e-300)).argmax()].item():.4f}"
