"""dspark_rms_norm_quant's ring of rows when its waits run out: with the diagnostic poll limit at "no poll at all" every
thread gives up its first wait, at one poll some do; a thread that gave up reads its part of the rows from memory, so the
outputs are bit for bit those of the ordinary call, and the copies asked for have landed before a CTA leaves."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu


def run(x, w, residual, n_live, in_place):
    x = x.clone()
    n, d = x.shape
    r = None if residual is None else residual.clone()
    h = None if r is None else (r if in_place else torch.empty_like(x))
    y = x if in_place else torch.zeros_like(x)
    q = torch.full((n, d), 55, dtype=torch.int8, device="cuda")
    s = torch.full((n,), -9.0, device="cuda")
    B.dspark_rms_norm_quant(x, w, 1e-6, residual=r, out_residual=h, out_q=q, out_scale=s, out_norm=y, n_live=n_live)
    torch.cuda.synchronize()
    return [t for t in (q, s, y, h) if t is not None]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", [(700, 1032), (3000, 2048), (650, 8200), (5000, 256), (9000, 64), (5000, 1000)])
@pytest.mark.parametrize("with_residual,live,in_place", [(True, None, False), (True, None, True), (False, 4771, False)])
def test_waits_that_run_out(dtype, n, d, with_residual, live, in_place):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    x[n // 2] = 0
    x[n // 3] = 1e-36                           # a row done after the last one
    r = torch.randn(n, d, generator=g, device="cuda").to(dtype) if with_residual else None
    w = torch.randn(d, generator=g, device="cuda").to(dtype)
    n_live = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
    want = run(x, w, r, n_live, in_place)
    for polls in (1, 2, 3):
        B.dspark_set_wait_poll_limit(polls)
        try:
            got = run(x, w, r, n_live, in_place)
        finally:
            B.dspark_set_wait_poll_limit(0)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), polls
    assert all(torch.equal(a, b) for a, b in zip(run(x, w, r, n_live, in_place), want))
