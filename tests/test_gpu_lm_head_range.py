"""The weight quantiser at the ends of bf16's range."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [3e38, 1e37, 2.7e36, 1e36, 1.0, 1e-36, 1e-38, 1e-39, 1e-40])
@pytest.mark.parametrize("K", [1, 7, 256, 1000])
def test_quantise_any_size(size, K):
    # integers equal; the scale is one rounding of max / 127 (2^-24, or half of fp32's smallest subnormal number)
    g = torch.Generator(device="cuda").manual_seed(K)
    w = ((torch.rand(20, K, generator=g, device="cuda", dtype=torch.float64) * 2 - 1) * size).bfloat16()
    w[3] = 0
    q = torch.full((20, K + 2), 55, dtype=torch.int8, device="cuda")
    s = torch.empty(20, device="cuda")
    B.dspark_lm_head_quantize(w, q[:, :K], s)
    wd = w.double()
    top = wd.abs().amax(1, keepdim=True)
    want = torch.where(top > 0, torch.round(wd * 127 / torch.where(top > 0, top, 1.0)), 0.0)
    assert torch.equal(q[:, :K].double(), want) and (q[:, K:] == 55).all()
    assert ((s.double() - top[:, 0] / 127).abs() <= 2.0 ** -24 * top[:, 0] / 127 + 2.0 ** -150).all()


def test_halves_of_large_weights_go_to_the_even_integer():
    w = (torch.tensor([[254.0] + [2.0 * k + 1 for k in range(127)] + [-2.0 * k - 1 for k in range(127)]], dtype=torch.float64) * 2.0 ** 119).bfloat16().cuda()
    q, s = torch.empty(1, 255, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    B.dspark_lm_head_quantize(w, q, s)
    assert torch.equal(q.double(), torch.round(w.double() / 2.0 ** 120))
