"""dspark_rms_norm_quant on rows at the bottom of fp32's range: products h * weight that are subnormal or below, down to
what only 64 bits hold.

Tolerances.  Integers and the stored sum have to be equal.  The scale: 48 x 2^-24 of itself as for ordinary rows, and half
a unit of the smallest subnormal number (2^-150).  The normalised row: half a step of its type, and half of its own
smallest subnormal number (bf16 2^-134, fp32 2^-150).  In rows whose largest product is an ordinary number, (h w) rstd is
computed in fp32: an element whose product h w is subnormal is off by half a unit of it, 2^-150, times rstd (7e-13 of the
row's largest value at the most: that one is above 1e-33 rstd)."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu

SCALE_TOL = 48 * 2.0 ** -24


def reference(x, residual, w, eps):
    h = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    t = h.double() * w.double()
    top = t.abs().amax(1, keepdim=True)
    zero = top == 0
    q = torch.where(zero, 0.0, torch.round(t * 127 / torch.where(zero, 1.0, top)))
    rstd = 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps)
    y = torch.where(zero, 0.0, t * torch.where(zero, 1.0, rstd))
    return h, q.to(torch.int8), y.abs().amax(1) / 127, y, torch.where(top >= 1e-33, rstd, 0.0)


def check(x, w, eps, residual, in_place=False):
    n, d = x.shape
    rh, rq, rs, ry, rstd = reference(x, residual, w, eps)
    h = (residual if in_place else torch.empty_like(x)) if residual is not None else None
    y = x if in_place else torch.empty_like(x)
    q = torch.full((n, d), 55, dtype=torch.int8, device="cuda")
    s = torch.full((n,), -9.0, device="cuda")
    B.dspark_rms_norm_quant(x, w, eps, residual=residual, out_residual=h, out_q=q, out_scale=s, out_norm=y)
    torch.cuda.synchronize()
    if h is not None:
        assert torch.equal(h, rh)
    assert torch.equal(q, rq)
    assert ((s.double() - rs).abs() <= SCALE_TOL * rs + 2.0 ** -150).all()
    half, least = torch.finfo(x.dtype).eps / 2, (2.0 ** -134 if x.dtype == torch.bfloat16 else 2.0 ** -150)
    assert ((y.double() - ry).abs() <= (half + SCALE_TOL) * 1.01 * ry.abs() + 1.01 * least + 2.0 ** -150 * rstd).all()


# element by element, a warp a row, a CTA a row, rings of rows by CTA and by warp
SIZES = [(3, 7), (5, 255), (4, 256), (2, 4096), (1, 5001), (2, 16384), (1300, 512), (600, 1032), (4800, 1000), (593, 16384)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", SIZES)
@pytest.mark.parametrize("with_residual", [True, False])
def test_tiny_products(dtype, n, d, with_residual):
    g = torch.Generator(device="cuda").manual_seed(n + 7 * d)
    # one size of product a row: 1e-31 (ordinary) to 1e-60; h is kept above 1e-30, the weights carry the rest
    size = torch.linspace(-31, -46, n, device="cuda") if n > 8 else torch.tensor([-43.0, -38.0, -40.5, -60.0, -33.1], device="cuda")[:n]
    at_w = -30.0
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).double() * 10.0 ** at_w
    x = torch.randn(n, d, generator=g, device="cuda").double() * (10.0 ** (size.double() - at_w))[:, None]
    r = (torch.randn(n, d, generator=g, device="cuda").double() * (10.0 ** (size.double() - at_w))[:, None]).to(dtype) if with_residual else None
    check(x.to(dtype), w.to(dtype), 1e-6, r)


@pytest.mark.parametrize("n,d", [(3, 63), (4, 4096), (600, 2048), (5000, 256)])
def test_tiny_products_in_place(n, d):
    g = torch.Generator(device="cuda").manual_seed(n)
    w = (torch.randn(d, generator=g, device="cuda") * 1e-25).bfloat16()
    x = (torch.randn(n, d, generator=g, device="cuda") * 1e-16).bfloat16()
    r = (torch.randn(n, d, generator=g, device="cuda") * 1e-16).bfloat16()
    x[n // 2] = 0
    r[n // 2] = 0
    check(x, w, 1e-6, r, in_place=True)


@pytest.mark.parametrize("dtype,h,w", [(torch.float32, 2e-25, 1e-20), (torch.float32, 1.0143e-23, 1e-20), (torch.bfloat16, 1.0987e-23, 1e-20),
                                       (torch.float32, 1e-45, 1.0), (torch.bfloat16, 1e-40, 0.5)])
def test_the_largest_product_is_127(dtype, h, w):
    x = torch.tensor([[h, -h, 0.0, h / 2]], dtype=torch.float64).to(dtype).cuda()
    ww = torch.full((4,), w, dtype=torch.float64).to(dtype).cuda()
    q, s = torch.empty(1, 4, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    B.dspark_rms_norm_quant(x, ww, 1e-6, out_q=q, out_scale=s)
    assert q[0, :3].tolist() == [127, -127, 0]
