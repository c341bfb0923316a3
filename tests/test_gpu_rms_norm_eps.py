"""dspark_rms_norm_quant on rows whose squares underflow in fp32, with an eps of zero or one that is as small, and on rows of
zeros.  Tolerances: those of the rows with tiny products."""
import pytest
import torch

from test_gpu_rms_norm_tiny import SIZES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", SIZES)
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-44])
def test_squares_that_underflow(dtype, n, d, eps):
    g = torch.Generator(device="cuda").manual_seed(n + 11 * d)
    size = torch.linspace(-14, -44, n, device="cuda") if n > 8 else torch.tensor([-19.0, -25.0, -22.3, -38.0, -18.0], device="cuda")[:n]
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    x = (torch.randn(n, d, generator=g, device="cuda").double() * (10.0 ** size.double())[:, None]).to(dtype)
    # rows this small can round to nothing but zeros in bf16; the reference knows.  eps as the call takes it, in fp32
    check(x, w, float(torch.tensor(eps, dtype=torch.float32)), None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", [(2, 5), (2, 4096), (700, 2048), (5000, 128)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_of_zeros(dtype, n, d, eps):
    x = torch.zeros(n, d, dtype=dtype, device="cuda")
    x[0] = -0.0
    w = torch.randn(d, device="cuda").to(dtype)
    check(x, w, eps, None)
    check(torch.ones_like(x), torch.zeros_like(w), eps, None)
