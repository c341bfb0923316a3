"""dspark_rms_norm_quant against the formula in 64 bits.

Tolerances.  The stored sum and the integers have to be equal: the sum is one rounding, the integers are those of the
exact quotient (the reference divides the exact products in 64 bits).  The scale: a thread adds at most 64 squares one
after the other and ten shuffles follow, each within 2^-24 of a sum of positive terms; the square root halves that
(37 x 2^-24); mean, root, reciprocal and three products add at most one rounding each: 48 x 2^-24.  The normalised row
adds its own rounding to the output type."""
import numpy as np
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu

SCALE_TOL = 48 * 2.0 ** -24


def reference(x, residual, w, eps):
    h = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    t = h.double() * w.double()
    top = t.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(t * 127 / top), torch.zeros_like(t))
    rstd = 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps)
    return h, q.to(torch.int8), (top * rstd / 127)[:, 0], t * rstd


def call(x, w, eps=1e-6, residual=None, n_live=None, want_norm=True, pads=(0, 0, 0)):
    n, d = x.shape
    h = torch.full((n, d + pads[0]), 7.0, dtype=x.dtype, device="cuda")
    q = torch.full((n, d + pads[1]), 55, dtype=torch.int8, device="cuda")
    y = torch.full((n, d + pads[2]), -3.0, dtype=x.dtype, device="cuda")
    s = torch.full((n,), -9.0, device="cuda")
    B.dspark_rms_norm_quant(x, w, eps, residual=residual, out_residual=h[:, :d], out_q=q[:, :d], out_scale=s,
                            out_norm=y[:, :d] if want_norm else None, n_live=n_live)
    torch.cuda.synchronize()
    return h, q, s, y


def check(x, w, eps, residual, got, live=None):
    n, d = x.shape
    live = n if live is None else live
    h, q, s, y = got
    rh, rq, rs, ry = reference(x, residual, w, eps)
    assert torch.equal(h[:live, :d], rh[:live])
    assert torch.equal(q[:live, :d], rq[:live])
    assert ((s[:live].double() - rs[:live]).abs() <= SCALE_TOL * rs[:live]).all()
    half = torch.finfo(x.dtype).eps / 2
    assert ((y[:live, :d].double() - ry[:live]).abs() <= (half + SCALE_TOL) * 1.01 * ry[:live].abs() + 1e-40).all()
    # nothing outside the rows that count or beyond their width
    assert (h[live:] == 7).all() and (q[live:] == 55).all() and (y[live:] == -3).all() and (s[live:] == -9).all()
    assert (h[:, d:] == 7).all() and (q[:, d:] == 55).all() and (y[:, d:] == -3).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", [(1, 1), (1, 7), (3, 64), (5, 255), (2, 1000), (2, 1024), (4, 1025), (3, 1032), (2, 4096), (1, 5000),
                                 (2, 8200), (1, 16383), (2, 16384), (1300, 512), (1187, 72)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_sizes(dtype, n, d, with_residual):
    g = torch.Generator(device="cuda").manual_seed(n * 100003 + d)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    r = (3 * torch.randn(n, d, generator=g, device="cuda")).to(dtype) if with_residual else None
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    check(x, w, 1e-6, r, call(x, w, 1e-6, r))


# many rows: rings of rows in shared memory, a CTA or a warp per row
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", [(600, 1032), (1500, 4096), (700, 8192), (593, 16384), (650, 10000), (5000, 512), (4800, 1000), (6001, 24), (9000, 264)])
@pytest.mark.parametrize("with_residual,live", [(True, None), (False, None), (True, 595), (False, 4737)])
def test_many_rows(dtype, n, d, with_residual, live):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    x[n // 2] = 0
    x[n // 3, d - 1] = float("nan")
    r = (3 * torch.randn(n, d, generator=g, device="cuda")).to(dtype) if with_residual else None
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    got = call(x, w, 1e-6, r, n_live=None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda"), pads=(8, 16, 8))
    rows = n if live is None else min(live, n)
    assert torch.isnan(got[2][n // 3]) if n // 3 < rows else True
    # the row with the NaN apart, everything as the formula says
    keep = torch.arange(n, device="cuda") != n // 3
    check(x[keep], w, 1e-6, r[keep] if with_residual else None, tuple(t[keep] for t in got), live=rows - (1 if n // 3 < rows else 0))


@pytest.mark.parametrize("n,d", [(3000, 2048), (5000, 256)])
def test_many_rows_in_place(n, d):
    x = torch.randn(n, d, device="cuda").bfloat16()
    r = torch.randn(n, d, device="cuda").bfloat16()
    w = torch.randn(d, device="cuda").bfloat16()
    rh, rq, rs, ry = reference(x, r, w, 1e-6)
    q = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s = torch.empty(n, device="cuda")
    B.dspark_rms_norm_quant(x, w, 1e-6, residual=r, out_residual=r, out_q=q, out_scale=s, out_norm=x)
    assert torch.equal(r, rh) and torch.equal(q, rq)
    assert ((x.double() - ry).abs() <= (2.0 ** -8 + SCALE_TOL) * 1.01 * ry.abs()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad_in,pads,offset", [(8, (8, 16, 24), 0), (1, (0, 0, 0), 0), (0, (1, 0, 0), 0), (0, (0, 3, 0), 0), (0, (0, 0, 5), 0), (8, (8, 8, 8), 1)])
def test_strides_and_alignment(dtype, pad_in, pads, offset):
    n, d = 6, 1032
    g = torch.Generator(device="cuda").manual_seed(5)
    full = torch.randn(n, d + pad_in + offset, generator=g, device="cuda").to(dtype)
    x = full[:, offset: offset + d]
    r = torch.randn(n, d + pad_in, generator=g, device="cuda").to(dtype)[:, :d]
    w = torch.randn(d, generator=g, device="cuda").to(dtype)
    check(x, w, 1e-5, r, call(x, w, 1e-5, r, pads=pads))


def test_halves_go_to_the_even_integer():
    # products at odd multiples of top / 254: the quotient is exactly a half
    top = 254.0
    x = torch.tensor([[top] + [float(2 * k + 1) for k in range(127)] + [-float(2 * k + 1) for k in range(127)]], device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        xx = x.to(dtype)
        assert torch.equal(xx.float(), x)
        w = torch.ones(x.shape[1], dtype=dtype, device="cuda")
        _, q, _, _ = call(xx, w)
        want = torch.round(x.double() / 2).to(torch.int8)
        assert torch.equal(q, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_neighbouring_values_next_to_a_half(dtype):
    # every bf16 value within a few steps of the halves of an awkward maximum
    top = torch.tensor(193.0).to(dtype)
    base = [(k + 0.5) * 193 / 127 for k in range(127)]
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    vals = [b * (1 + s * eps) for b in base for s in (-2, -1, 0, 1, 2)]
    x = torch.tensor([[193.0] + vals]).to(dtype).cuda()
    w = torch.ones(x.shape[1], dtype=dtype, device="cuda")
    check(x, w, 1e-6, None, call(x, w))
    assert float(top) == 193.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [40, 4096])
def test_special_rows(dtype, d):
    x = torch.randn(9, d, device="cuda").to(dtype)
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, d - 1] = float("inf")
    x[3, 5] = float("-inf")
    x[4] = 3e19                       # squares pass fp32's range
    x[5] = 1e-30                      # squares underflow: the norm is eps alone
    x[6] = -0.0
    x[7, 2:] = 0
    w = torch.ones(d, dtype=dtype, device="cuda")
    h, q, s, y = call(x, w)
    assert float(s[0]) == 0 and (q[0] == 0).all()
    assert float(s[6]) == 0 and (q[6] == 0).all()
    for r in (1, 2, 3, 4):
        assert torch.isnan(s[r]) and (q[r] == 0).all()
    good = [0, 5, 6, 7, 8]
    _, rq, rs, _ = reference(x[good], None, w, 1e-6)
    assert torch.equal(q[good], rq)
    assert ((s[good].double() - rs).abs() <= SCALE_TOL * rs).all()
    wn = w.clone()
    wn[1] = float("nan")
    _, q, s, _ = call(torch.ones(2, d, dtype=dtype, device="cuda"), wn)
    assert torch.isnan(s).all() and (q == 0).all()


@pytest.mark.parametrize("live", [0, 1, 5, 12, 40])
def test_rows_behind_the_last_one_are_left(live):
    n, d = 12, 2048
    x = torch.randn(n, d, device="cuda").bfloat16()
    r = torch.randn(n, d, device="cuda").bfloat16()
    w = torch.randn(d, device="cuda").bfloat16()
    got = call(x, w, 1e-6, r, n_live=torch.tensor([live], dtype=torch.int32, device="cuda"))
    check(x, w, 1e-6, r, got, live=min(live, n))


def test_in_place():
    n, d = 17, 1536
    x = torch.randn(n, d, device="cuda").bfloat16()
    r = torch.randn(n, d, device="cuda").bfloat16()
    w = torch.randn(d, device="cuda").bfloat16()
    rh, rq, rs, ry = reference(x, r, w, 1e-6)
    q = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s = torch.empty(n, device="cuda")
    B.dspark_rms_norm_quant(x, w, 1e-6, residual=r, out_residual=r, out_q=q, out_scale=s, out_norm=x)
    assert torch.equal(r, rh) and torch.equal(q, rq)
    assert ((x.double() - ry).abs() <= (2.0 ** -8 + SCALE_TOL) * 1.01 * ry.abs()).all()
